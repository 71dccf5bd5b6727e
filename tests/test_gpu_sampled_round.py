"""A whole decoding round of the operators together -- heads normalised, rotated and placed, attention with shaped scores,
sampled verification, compaction -- on a paged and on a contiguous cache, against the oracles' chain."""
import numpy as np
import pytest
import torch

from oracle import place_oracle as po
from oracle import sample_oracle as so
from oracle import scored_oracle as sc

pytestmark = pytest.mark.gpu


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("ps", [0, 16], ids=["contiguous", "paged"])
def test_two_rounds(oracle, ps):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2404_12022_b200 import binding as hb
    dt, B, T, P, Hq, Hkv, D, V, per = torch.bfloat16, 3, 20, 3, 8, 4, 128, 500, 20
    N, cap = T + P, per * 16
    g = torch.Generator().manual_seed(77)
    rnd = lambda *s: torch.randn(s, generator=g)                                        # noqa: E731
    rng = np.random.default_rng(77)
    parent = np.full((B, N), -1, np.int32)
    depth = np.zeros((B, N), np.int32)
    for b in range(B):
        for r in range(1, N):
            parent[b, r] = rng.integers(0, r) if r < T else (r - 1 if r > T else 4)
            depth[b, r] = depth[b, parent[b, r]] + 1
    lens = np.array([0, 100, 250], np.int32)
    kc, vc = (rnd(B, Hkv, cap, D).to(dt).cuda() for _ in range(2))
    table = None
    if ps:
        table = torch.randperm(B * per + 1, generator=g)[:B * per].int().view(B, per).cuda()
        pools = []
        for t in (kc, vc):
            pool = torch.zeros((B * per + 1, Hkv, ps, D), dtype=dt, device="cuda")
            pool[table.long().flatten()] = t.view(B, Hkv, per, ps, D).permute(0, 2, 1, 3, 4).reshape(-1, Hkv, ps, D)
            pools.append(pool)
        kc, vc = pools
    view = (lambda t: t[table.long()].permute(0, 2, 1, 3, 4).reshape(B, Hkv, cap, D)) if ps else (lambda t: t)
    qw, kw = (1 + 0.2 * rnd(D)).to(dt).cuda(), (1 + 0.2 * rnd(D)).to(dt).cuda()
    head = hb.make_head_desc(D, rot_dim=64, interleaved=True, scaling=hb.HT_ROPE_LINEAR, factor=2.0)
    slopes = torch.tensor([2.0 ** -(h + 1) for h in range(Hq)], device="cuda")
    par = torch.from_numpy(parent).cuda()
    kv_len = torch.from_numpy(lens).cuda()
    root = torch.randint(0, V, (B,), generator=g).int().cuda()
    top_p, temp = torch.full((B,), 0.9, device="cuda"), torch.full((B,), 0.8, device="cuda")
    accept_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    for _ in range(2):
        pos = torch.from_numpy(kv_len.cpu().numpy()[:, None] + depth).int().cuda()
        qkv = rnd(B, N, (Hq + 2 * Hkv) * D).to(dt).cuda()
        q, k, v = (t.unflatten(2, (-1, D)) for t in qkv.split([Hq * D, Hkv * D, Hkv * D], 2))
        before = f64(view(kc)), f64(view(vc))
        at = kv_len.cpu().numpy()
        if ps:
            qo, st = hb.norm_rope_kv_append_paged(q, k, v, pos, kv_len, table, kc, vc, head, qw, kw)
            out, st2 = hb.tree_attention_scored_paged(qo, kc, vc, table, kv_len, par, cap=20.0, slopes=slopes, pos=pos)
        else:
            qo, st = hb.norm_rope_kv_append(q, k, v, pos, kv_len, kc, vc, head, qw, kw)
            out, st2 = hb.tree_attention_scored(qo, kc, vc, kv_len, par, cap=20.0, slopes=slopes, pos=pos)
        assert (st == 0).all() and (st2 == 0).all()
        # rows placed: one rounding (2^-9 relative; 2^-8 covers the arithmetic) on a head's largest value
        rk = po.heads(f64(k), pos.cpu().numpy(), f64(kw), rot_dim=64, interleaved=True, scaling="linear", factor=2.0)
        K, Vc = f64(view(kc)), f64(view(vc))
        for b in range(B):
            L = at[b]
            assert np.abs(K[b, :, L:L + N].swapaxes(0, 1) - rk[b]).max() <= 2.0 ** -8 * np.abs(rk[b]).max()
            assert np.array_equal(Vc[b, :, L:L + N].swapaxes(0, 1), f64(v)[b]) and np.array_equal(K[b, :, :L], before[0][b, :, :L])
        # attention over what the cache now holds: the bound of the plain entry point
        ref = sc.tree_attention(f64(qo), K, Vc, at, parent, 20.0, f64(slopes), pos.cpu().numpy())
        assert (np.abs(f64(out) - ref) <= 2e-3 + 1e-2 * np.abs(ref)).all()
        # logits that stand in for the rest of the model, drafts that mostly follow the samples
        x = (3 * rnd(B, N, V)).to(dt).cuda()
        u = torch.rand((B, N), generator=g).cuda()
        drawn = so.sample(f64(x)[:, :T], f64(u), f64(temp), None, f64(top_p))
        tokens = rng.integers(0, V, (B, T)).astype(np.int32)
        for b in range(B):
            for c in range(T):
                if rng.random() < 0.8:
                    tokens[b, c] = int(root[b]) if parent[b, c] < 0 else drawn[b, parent[b, c]]
        pred, alen, path, nxt, vst = hb.verify_sampled(x, u, torch.from_numpy(tokens).cuda(), par, root, temp, None, top_p, None, 16, accept_len)
        full = np.full((B, N), -1, np.int32)
        full[:, :T] = drawn
        want = oracle.accept_scan(tokens, parent, full, root.cpu().numpy(), 16)
        for a, w in zip((pred, alen, path, nxt, vst), (full, *want)):
            assert np.array_equal(a.cpu().numpy(), w)
        # the accepted path's rows follow the context
        if ps:
            new_len, cst = hb.kv_compact_paged(kc[None], vc[None], table, N, kv_len, alen, path)
        else:
            new_len, cst = hb.kv_compact(kc[None], vc[None], N, kv_len, alen, path)
        assert (cst == 0).all() and np.array_equal(new_len.cpu().numpy(), at + want[0])
        for b in range(B):
            rows = at[b] + want[1][b, :want[0][b]]
            assert np.array_equal(f64(view(kc))[b, :, at[b]:at[b] + want[0][b]], K[b][:, rows])
        kv_len, root = new_len, nxt


@pytest.mark.parametrize("ps", [0, 16], ids=["contiguous", "paged"])
def test_rounds_leave_every_row_where_it_belongs(ps):
    """Keys and values alike, the rows ahead of the tree included, and attention held to the bound of its own tests."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2404_12022_b200 import binding as hb
    from test_gpu_scored_attention import close
    dt, B, T, N, Hq, Hkv, D, V, per = torch.float16, 3, 12, 14, 4, 2, 128, 50, 8
    cap = per * 16
    g = torch.Generator().manual_seed(78)
    rnd = lambda *s: torch.randn(s, generator=g).to(dt).cuda()                          # noqa: E731
    rng = np.random.default_rng(78)
    parent = np.full((B, N), -1, np.int32)
    depth = np.zeros((B, N), np.int32)
    for b in range(B):
        for r in range(1, N):
            parent[b, r] = rng.integers(max(0, r - 3), r) if r < T else 2
            depth[b, r] = depth[b, parent[b, r]] + 1
    kc, vc = rnd(B, Hkv, cap, D), rnd(B, Hkv, cap, D)
    table = None
    if ps:
        table = torch.randperm(B * per + 1, generator=g)[:B * per].int().view(B, per).cuda()
        pools = []
        for t in (kc, vc):
            pool = torch.zeros((B * per + 1, Hkv, ps, D), dtype=dt, device="cuda")
            pool[table.long().flatten()] = t.view(B, Hkv, per, ps, D).permute(0, 2, 1, 3, 4).reshape(-1, Hkv, ps, D)
            pools.append(pool)
        kc, vc = pools
    view = (lambda t: t[table.long()].permute(0, 2, 1, 3, 4).reshape(B, Hkv, cap, D)) if ps else (lambda t: t)
    head = hb.make_head_desc(D)
    slopes = torch.tensor([0.5, 0.1, 0.02, 0.0], device="cuda")
    par, kv_len = torch.from_numpy(parent).cuda(), torch.tensor([0, 17, 60], dtype=torch.int32, device="cuda")
    accept_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    moved = 0
    for _ in range(3):
        at = kv_len.cpu().numpy()
        pos = torch.from_numpy(at[:, None] + depth).int().cuda()
        q, k, v = rnd(B, N, Hq, D), rnd(B, N, Hkv, D), rnd(B, N, Hkv, D)
        before = f64(view(kc)), f64(view(vc))
        if ps:
            qo, st = hb.norm_rope_kv_append_paged(q, k, v, pos, kv_len, table, kc, vc, head)
            out, st2 = hb.tree_attention_scored_paged(qo, kc, vc, table, kv_len, par, cap=25.0, slopes=slopes, pos=pos)
        else:
            qo, st = hb.norm_rope_kv_append(q, k, v, pos, kv_len, kc, vc, head)
            out, st2 = hb.tree_attention_scored(qo, kc, vc, kv_len, par, cap=25.0, slopes=slopes, pos=pos)
        assert (st == 0).all() and (st2 == 0).all()
        placed = f64(view(kc)), f64(view(vc))
        close(out, sc.tree_attention(f64(qo), *placed, at, parent, 25.0, f64(slopes), pos.cpu().numpy(), spread=True))
        x, u = rnd(B, N, V), torch.rand((B, N), generator=g).cuda()
        drawn = so.sample(f64(x)[:, :T], f64(u))
        tokens = rng.integers(0, V, (B, T)).astype(np.int32)
        for b in range(B):
            for c in range(1, T):
                if rng.random() < 0.9:
                    tokens[b, c] = drawn[b, parent[b, c]]
        _, alen, path, _, vst = hb.verify_sampled(x, u, torch.from_numpy(tokens).cuda(), par, max_path=12, accept_len=accept_len)
        if ps:
            new_len, cst = hb.kv_compact_paged(kc[None], vc[None], table, N, kv_len, alen, path)
        else:
            new_len, cst = hb.kv_compact(kc[None], vc[None], N, kv_len, alen, path)
        assert (vst == 0).all() and (cst == 0).all()
        n, p = alen.cpu().numpy(), path.cpu().numpy()
        assert np.array_equal(new_len.cpu().numpy(), at + n)
        for now, mid, old in zip((f64(view(kc)), f64(view(vc))), placed, before):
            for b in range(B):
                L = at[b]
                moved += (p[b, :n[b]] != np.arange(n[b])).sum()
                assert np.array_equal(now[b, :, :L], old[b, :, :L])                     # the context
                assert np.array_equal(now[b, :, L:L + n[b]], mid[b][:, L + p[b, :n[b]]])      # the accepted path behind it
                assert np.array_equal(now[b, :, L + N:], old[b, :, L + N:])             # rows behind the tree
        assert np.array_equal(placed[1][0][:, at[0]:at[0] + N], f64(v)[0].swapaxes(0, 1))
        kv_len = new_len
    assert moved > 0                                          # (paths that skip nodes have been moved)
