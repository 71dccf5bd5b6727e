"""Norm + rotary + cache append on the GPU against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import place_oracle as po

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def hb():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2404_12022_b200 import binding
    binding.load()
    return binding


def f64(t):
    return t.double().cpu().numpy()


def close(got, ref, what=""):
    """One rounding to the type, half a step relative (eps / 2), and what 32-bit arithmetic adds: the sum of D <= 128 squares in
    a tree (about 20 roundings), root, quotient, two products, and for a rotated pair four more on values up to the head's
    largest, with cosine and sine off by about 2^-23: below 48 * 2^-24 of the head's largest value.  Subnormal results are
    off by half the smallest step."""
    g = f64(got)
    big = np.abs(ref).max(-1, keepdims=True)
    info = torch.finfo(got.dtype)
    arith = 48 * 2.0 ** -24 * big
    tol = info.eps / 2 * (np.abs(ref) + arith) + arith + info.smallest_normal * info.eps / 2
    bad = np.abs(g - ref) > tol
    assert not bad.any(), "%s: %d of %d off, worst %.3g" % (what, bad.sum(), bad.size, (np.abs(g - ref) - tol).max())


def case(seed, dt, B, N, Hq, Hkv, D, fused=True):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g)                                        # noqa: E731
    width = (Hq + 2 * Hkv) * D
    if fused:                                                                          # one buffer, rows width + 16 apart
        buf = rnd(B, N, width + 16).to(dt).cuda()
        q, k, v = buf[..., :Hq * D], buf[..., Hq * D:(Hq + Hkv) * D], buf[..., (Hq + Hkv) * D:width]
        q, k, v = q.unflatten(2, (Hq, D)), k.unflatten(2, (Hkv, D)), v.unflatten(2, (Hkv, D))
    else:
        q, k, v = (rnd(B, N, h, D).to(dt).cuda() for h in (Hq, Hkv, Hkv))
    qw, kw = (1 + 0.3 * rnd(D)).to(dt).cuda(), (1 + 0.3 * rnd(D)).to(dt).cuda()
    pos = torch.randint(0, 120000, (B, N), generator=g).int().cuda()
    return q, k, v, qw, kw, pos


HEADS = [dict(), dict(rot_dim=0), dict(interleaved=True), dict(rot_dim=32), dict(interleaved=True, rot_dim=22, weight_offset=1.0),
         dict(scaling="linear", factor=4.0, rope_base=500000.0), dict(interleaved=True, rot_dim=2, eps=1e-2),
         dict(scaling="parts", factor=8.0, orig_len=8192.0, low=1.0, high=4.0, rope_base=500000.0, magnitude=1.2)]


def run_one(hb, dt, shape, kw, fused, norm, in_place=False):
    B, N, Hq, Hkv, D = shape
    q, k, v, qw, kwt, pos = case(11, dt, B, N, Hq, Hkv, D, fused)
    cap = N + 37
    kc, vc = (torch.full((B, Hkv, cap, D), 7.0, dtype=dt, device="cuda") for _ in range(2))
    lens = np.array([(13 * b) % 38 for b in range(B)], np.int32)
    scaling = kw.get("scaling", "plain")
    hkw = {k_: v_ for k_, v_ in kw.items() if k_ != "scaling"}
    head = hb.make_head_desc(D, norm=norm, scaling={"plain": 0, "linear": 1, "parts": 2}[scaling], **hkw)
    okw = dict(hkw)
    okw["offset"] = okw.pop("weight_offset", 0.0)
    okw["base"] = okw.pop("rope_base", 10000.0)
    okw["scaling"] = scaling
    q0, k0, v0, p0 = f64(q), f64(k), f64(v), pos.cpu().numpy()
    out, st = hb.norm_rope_kv_append(q, k, v, pos, torch.from_numpy(lens).cuda(), kc, vc, head, qw, kwt, q_out=q if in_place else None)
    assert (st.cpu().numpy() == 0).all()
    close(out, po.heads(q0, p0, f64(qw), bool(norm & 1), **okw), "q")
    rk = po.heads(k0, p0, f64(kwt), bool(norm & 2), **okw)
    for b in range(B):
        L = int(lens[b])
        close(kc[b, :, L:L + N].transpose(0, 1), rk[b], "k")
        assert np.array_equal(f64(vc[b, :, L:L + N].transpose(0, 1)), v0[b])
        for c in (kc, vc):                                                             # nothing else is touched
            assert (c[b, :, :L] == 7).all() and (c[b, :, L + N:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 64), (2, 5, 6, 2, 128), (3, 18, 8, 8, 64), (2, 33, 72, 8, 128)],
                         ids=lambda s: "B%dN%dHq%dHkv%dD%d" % s)
@pytest.mark.parametrize("kw", HEADS, ids=lambda k: "_".join(k) or "plain")
def test_norm_rope_against_the_oracle(hb, dtype, shape, kw):
    run_one(hb, DT[dtype], shape, kw, fused=True, norm=3)


@pytest.mark.parametrize("dtype,shape", [("bf16", (1, 5, 128, 32, 128)), ("f32", (2, 3, 128, 32, 128)), ("f16", (8, 400, 2, 1, 64)),
                                         ("bf16", (3, 700, 33, 3, 128))], ids=lambda s: str(s))
def test_more_heads_than_a_block_takes_and_more_rows_than_blocks(hb, dtype, shape):
    run_one(hb, DT[dtype], shape, dict(rot_dim=64), fused=True, norm=3)


@pytest.mark.parametrize("norm", [0, 1, 2])
def test_norm_of_either_side_dense_inputs_and_in_place(hb, norm):
    run_one(hb, torch.bfloat16, (2, 9, 8, 4, 128), {}, fused=False, norm=norm)
    run_one(hb, torch.float16, (2, 9, 8, 4, 128), dict(interleaved=True), fused=False, norm=norm, in_place=True)


def test_plain_rotation_is_what_rope_kv_append_gives(hb):
    """Without norms the operation is that of ht_rope_kv_append: two results of one formula, each within its bound."""
    dt, (B, N, Hq, Hkv, D) = torch.bfloat16, (2, 19, 8, 4, 128)
    q, k, v, _, _, pos = case(3, dt, B, N, Hq, Hkv, D, fused=False)
    lens = torch.tensor([3, 30], dtype=torch.int32, device="cuda")
    caches = [torch.zeros((B, Hkv, 64, D), dtype=dt, device="cuda") for _ in range(4)]
    a, _ = hb.rope_kv_append(q, k, v, pos, lens, caches[0], caches[1])
    b, _ = hb.norm_rope_kv_append(q, k, v, pos, lens, caches[2], caches[3], hb.make_head_desc(D, norm=0))
    assert (a.float() - b.float()).abs().max() <= 2 * 2.0 ** -8 * a.float().abs().max()
    assert torch.equal(caches[1], caches[3])


def test_weights_may_be_left_out_and_infinities_stay_in_their_pair(hb):
    dt, D = torch.float32, 64
    q, k, v, _, _, pos = case(4, dt, 1, 2, 2, 2, D, fused=False)
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    kc, vc = (torch.zeros((1, 2, 8, D), dtype=dt, device="cuda") for _ in range(2))
    out, _ = hb.norm_rope_kv_append(q, k, v, pos, lens, kc, vc, hb.make_head_desc(D))
    close(out, po.heads(f64(q), pos.cpu().numpy()))
    for il in (False, True):
        q[0, 0, 0, 40] = float("inf")
        out, _ = hb.norm_rope_kv_append(q, k, v, pos, lens, kc, vc, hb.make_head_desc(D, norm=0, rot_dim=32, interleaved=il))
        assert out[0, 0, 0, 40] == float("inf") and torch.isfinite(out[0, 0, 0, :40]).all() and torch.isfinite(out[0, 0, 0, 41:]).all()


def test_bad_lengths_are_flagged_and_skipped(hb):
    dt, (B, N, H, D) = torch.float16, (4, 6, 2, 128)
    q, k, v, qw, kw, pos = case(5, dt, B, N, H, H, D)
    kc, vc = (torch.full((B, H, 16, D), 7.0, dtype=dt, device="cuda") for _ in range(2))
    q_out = torch.full((B, N, H, D), 5.0, dtype=dt, device="cuda")
    lens = torch.tensor([-1, 10, 11, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    out, st = hb.norm_rope_kv_append(q, k, v, pos, lens, kc, vc, hb.make_head_desc(D), qw, kw, q_out=q_out)
    assert st.tolist() == [2, 0, 2, 2]
    for b in (0, 2, 3):
        assert (kc[b] == 7).all() and (vc[b] == 7).all() and (out[b] == 5).all()
    assert (kc[1, :, 10:] != 7).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ps", [16, 64])
def test_paged_equals_contiguous_bit_for_bit(hb, dtype, ps):
    dt, (B, N, Hq, Hkv, D), cap = DT[dtype], (3, 37, 8, 4, 128), 192
    q, k, v, qw, kw, pos = case(6, dt, B, N, Hq, Hkv, D)
    lens = torch.tensor([0, 45, 192 - 37], dtype=torch.int32, device="cuda")
    head = hb.make_head_desc(D, rot_dim=64, interleaved=True, scaling=hb.HT_ROPE_LINEAR, factor=2.0)
    kc, vc = (torch.zeros((B, Hkv, cap, D), dtype=dt, device="cuda") for _ in range(2))
    want, _ = hb.norm_rope_kv_append(q, k, v, pos, lens, kc, vc, head, qw, kw)
    per = cap // ps
    table = torch.randperm(B * per + 3, generator=torch.Generator().manual_seed(1))[:B * per].int().view(B, per).cuda()
    pools = torch.zeros((2, 2, B * per + 3, Hkv, ps, D), dtype=dt, device="cuda")       # a view of a layer of a larger pool
    kp, vp = pools[0, 1], pools[1, 1]
    got, st = hb.norm_rope_kv_append_paged(q, k, v, pos, lens, table, kp, vp, head, qw, kw)
    assert torch.equal(got, want) and st.tolist() == [0, 0, 0]
    for pool, cache in ((kp, kc), (vp, vc)):
        assert torch.equal(pool[table.long()].permute(0, 2, 1, 3, 4).reshape(B, Hkv, cap, D), cache)
    assert (pools[:, 0] == 0).all()


def test_bad_pages_are_flagged_and_nothing_else_is_lost(hb):
    dt, (B, N, H, D), ps = torch.bfloat16, (3, 20, 2, 64), 16
    q, k, v, qw, kw, pos = case(7, dt, B, N, H, H, D)
    head = hb.make_head_desc(D)
    lens = torch.tensor([8, 8, 16], dtype=torch.int32, device="cuda")
    table = torch.tensor([[0, 1], [2, 99], [3, -5]], dtype=torch.int32, device="cuda")
    kp, vp = (torch.full((6, H, ps, D), 7.0, dtype=dt, device="cuda") for _ in range(2))
    out, st = hb.norm_rope_kv_append_paged(q, k, v, pos, lens, table, kp, vp, head, qw, kw)
    assert st.tolist() == [0, 5, 2]                                                     # the third does not fit its two pages
    close(out[:2], po.heads(f64(q), pos.cpu().numpy(), f64(qw))[:2])
    assert (kp[2, :, 8:] != 7).any() and (kp[3:] == 7).all()


def test_captured_and_replayed_on_new_inputs_and_on_another_stream(hb):
    dt, (B, N, Hq, Hkv, D) = torch.bfloat16, (2, 16, 8, 2, 128)
    q, k, v, qw, kw, pos = case(8, dt, B, N, Hq, Hkv, D)
    lens = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    kc, vc = (torch.zeros((B, Hkv, 32, D), dtype=dt, device="cuda") for _ in range(2))
    head = hb.make_head_desc(D)
    q_out = torch.empty((B, N, Hq, D), dtype=dt, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _, st = hb.norm_rope_kv_append(q, k, v, pos, lens, kc, vc, head, qw, kw, q_out=q_out)
    for seed in (1, 2):
        g = torch.Generator().manual_seed(seed)
        q.copy_(torch.randn(q.shape, generator=g).to(dt))
        pos.copy_(torch.randint(0, 5000, (B, N), generator=g).int())
        graph.replay()
        torch.cuda.synchronize()
        close(q_out, po.heads(f64(q), pos.cpu().numpy(), f64(qw)))


def test_binding_refuses_what_it_cannot_pass_on(hb):
    q, k, v, qw, kw, pos = case(9, torch.float16, 2, 4, 4, 2, 128)
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    kc = torch.zeros((2, 2, 16, 128), dtype=torch.float16, device="cuda")
    head = hb.make_head_desc(128)
    for bad in (dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(k=k.float()), dict(pos=pos.long()), dict(pos=pos[:1]), dict(qw=qw[:64]),
                dict(v=v[..., :64]), dict(lens=lens.cpu())):
        a = dict(q=q, k=k, v=v, pos=pos, lens=lens, qw=qw)
        a.update(bad)
        with pytest.raises(ValueError):
            hb.norm_rope_kv_append(a["q"], a["k"], a["v"], a["pos"], a["lens"], kc, kc.clone(), head, a["qw"], kw)
