"""Tree attention with capped and distance-biased scores on the GPU against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import scored_oracle as so

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
    """ref: the result o and A, the sums of weight * |v|, by the oracle.
    16-bit types: the tensor cores take the weights rounded to the type, each off by at most half a step, eps / 2 of itself
    (their sum is held in 32 bits): eps / 2 * A in all; a float16 weight below the type's range is lost or off by half
    its smallest step, which against the row's largest weight (at least 2^-8 of the running maximum's) is 2^-17 for all
    keys at most in the tests' lengths; the result is rounded once, eps / 2 * |o|; the scores' 32-bit sums of 128 products
    and the exponential move each weight by less than 2e-5 of itself.  Results of order one then differ by up to 6e-3 in
    bfloat16: tighter than this no such kernel can be held to, looser no result is let through.
    fp32: a score is a sum of 128 products (values to about 5 in all: rounding errors of 1e-6 at most in the mean square),
    the cap adds cap * 2^-23 (below 1e-5 for caps to 80) and the exponential 2^-22; an output moves by the score's error
    times a value spread of about one: 1e-5 (1 + |o|)."""
    o, size = ref
    g = f64(got)
    half = torch.finfo(got.dtype).eps / 2
    tol = 1e-5 * (1 + np.abs(o)) if got.dtype == torch.float32 else half * (size + np.abs(o)) + 2e-5 * size + 2.0 ** -17
    bad = np.abs(g - o) > tol
    assert not bad.any(), "%s: %d of %d off, worst %.3g" % (what, bad.sum(), bad.size, np.abs(g - o).max())


def case(seed, dtype, B, N, Hq, Hkv, D, lens, spread=2.0, slope=None):
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt = DT[dtype]
    cap = max(lens) + N + 5
    q = (spread * torch.randn((B, N, Hq, D), generator=g)).to(dt).cuda()
    k, v = (torch.randn((B, Hkv, cap, D), generator=g).to(dt).cuda() for _ in range(2))
    for b, L in enumerate(lens):                                                       # rows behind the tree are not data
        k[b, :, L + N:] = float("nan")
        v[b, :, L + N:] = float("inf")
    parent = np.full((B, N), -1, np.int32)
    depth = np.zeros((B, N), np.int32)
    for b in range(B):
        for r in range(1, N):
            parent[b, r] = rng.integers(max(-1, r - 7), r)
            depth[b, r] = depth[b, parent[b, r]] + 1 if parent[b, r] >= 0 else 0
    pos = np.asarray(lens, np.int32)[:, None] + depth
    slopes = 2.0 ** (-8.0 * np.arange(1, Hq + 1) / Hq) if slope is None else np.full(Hq, slope)
    dev = lambda a, t: torch.as_tensor(np.asarray(a), dtype=t).cuda()                   # noqa: E731
    return (q, k, v, dev(lens, torch.int32), dev(parent, torch.int32), dev(slopes, torch.float32), dev(pos, torch.int32))


def reference(c, cap, bias):
    q, k, v, lens, parent, slopes, pos = c
    return so.tree_attention(f64(q), f64(k), f64(v), lens.cpu().numpy(), parent.cpu().numpy(), cap, f64(slopes) if bias else None,
                             pos.cpu().numpy(), spread=True)


def check(hb, c, cap, bias, **kw):
    q, k, v, lens, parent, slopes, pos = c
    out, st = hb.tree_attention_scored(q, k, v, lens, parent, cap=cap, slopes=slopes if bias else None, pos=pos if bias else None, **kw)
    assert (st == 0).all()
    close(out, reference(c, cap, bias), "cap %g bias %s" % (cap, bias))


SHAPES = [(1, 1, 2, 2, 128, [0]), (1, 1, 4, 1, 128, [700]), (2, 18, 4, 4, 128, [130, 0]), (3, 40, 8, 2, 128, [127, 128, 333]),
          (2, 91, 4, 4, 128, [1000, 64]), (1, 67, 16, 2, 128, [515]), (1, 200, 4, 2, 128, [256]), (2, 18, 4, 4, 64, [31, 97]),
          (1, 24, 6, 2, 128, [200])]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "B%dN%dHq%dHkv%dD%d_%s" % (*s[:5], "_".join(map(str, s[5]))))
@pytest.mark.parametrize("cap,bias", [(30.0, False), (0.0, True), (4.0, True)], ids=["cap", "bias", "both"])
def test_scored_attention_against_the_oracle(hb, dtype, shape, cap, bias):
    check(hb, case(21, dtype, *shape), cap, bias)


@pytest.mark.parametrize("cap", [0.01, 1.0, 1000.0, 1e8])
def test_caps_from_saturated_to_hardly_there(hb, cap):
    """A cap of 0.01 flattens every score, one of 1e8 leaves them as they are (the series' result is taken there)."""
    for dtype in ("f32", "bf16"):
        c = case(22, dtype, 1, 30, 4, 2, 128, [300], spread=6.0)
        if dtype == "f32" and cap > 1000:
            continue                                  # tanhf's rounding times such a cap is what fp32 holds of the score
        check(hb, c, cap, False)


@pytest.mark.parametrize("slope", [3.0, 0.5, -0.01, 0.0])
def test_steep_flat_and_negative_slopes(hb, slope):
    for dtype in ("f16", "bf16", "f32"):
        check(hb, case(23, dtype, 2, 40, 4, 4, 128, [384, 200], slope=slope), 0.0, True)
    check(hb, case(24, "bf16", 1, 40, 16, 2, 128, [384], slope=slope), 0.0, True)


def test_nothing_asked_for_is_the_plain_call_bit_for_bit(hb):
    for shape in ((2, 18, 4, 4, 128, [130, 40]), (1, 67, 16, 2, 128, [515])):
        c = case(25, "bf16", *shape)
        a, _ = hb.tree_attention(*c[:5])
        b, _ = hb.tree_attention_scored(*c[:5])
        assert torch.equal(a, b)


@pytest.mark.parametrize("shape", [(1, 19, 8, 8, 128, [9000]), (1, 67, 64, 8, 128, [9000]), (8, 19, 40, 40, 128, [600, 20, 900, 333, 128, 1, 700, 512]),
                                   (4, 67, 16, 2, 128, [2000, 10, 1500, 800])], ids=lambda s: "B%dN%dHq%dHkv%d" % s[:4])
@pytest.mark.parametrize("final", [False, True], ids=["plain", "promises"])
def test_work_splits_clusters_and_promises(hb, shape, final):
    """Units cut over CTAs, clusters of every size, the tile-pair kernel; with a kept workspace and the early start."""
    c = case(26, "bf16", *shape)
    q, k, v, lens, parent, slopes, pos = c
    ws = torch.zeros(48 << 20, dtype=torch.uint8, device="cuda")
    flags = (hb.HT_ATTN_WORKSPACE_CLEAN | hb.HT_ATTN_CONTEXT_FINAL) if final else 0
    ref = reference(c, 30.0, True)
    for _ in range(2):
        out, st = hb.tree_attention_scored(q, k, v, lens, parent, cap=30.0, slopes=slopes, pos=pos, workspace=ws, flags=flags)
        assert (st == 0).all()
        close(out, ref)
    plain, _ = hb.tree_attention(q, k, v, lens, parent, workspace=ws, flags=flags)       # the two forms share a workspace
    close(plain, reference(c, 0.0, False))


@pytest.mark.parametrize("shape", [(1, 1000, 2, 2, 128, [64]), (1, 1024, 2, 1, 128, [0]), (2, 300, 4, 2, 128, [130, 5])],
                         ids=lambda s: "N%dHq%dHkv%d" % s[1:4])
def test_large_trees_on_strided_views_of_a_layered_cache(hb, shape):
    c = case(35, "bf16", *shape)
    q, k, v, lens, parent, slopes, pos = c
    layers = torch.zeros((2, 3) + tuple(k.shape), dtype=k.dtype, device="cuda")
    layers[0, 1], layers[1, 1] = k, v
    for cap, bias in ((10.0, False), (0.0, True), (10.0, True)):
        check(hb, (q, layers[0, 1], layers[1, 1], lens, parent, slopes, pos), cap, bias)


def test_waits_that_run_out_are_reported_and_leave_the_device_usable(hb):
    for shape in ((5, 37, 32, 32, 128, [900, 640, 33, 1200, 512]), (2, 19, 64, 8, 128, [3000, 2500])):
        c = case(36, "bf16", *shape)
        q, k, v, lens, parent, slopes, pos = c
        kw = dict(cap=20.0, slopes=slopes, pos=pos)
        _, st = hb.tree_attention_scored(q, k, v, lens, parent, flags=hb.HT_ATTN_TEST_SHORT_WAITS, **kw)
        assert all(s in (0, 6) for s in st.tolist()) and 6 in st.tolist()
        out, st = hb.tree_attention_scored(q, k, v, lens, parent, **kw)
        assert (st == 0).all()
        close(out, reference(c, 20.0, True))


@pytest.mark.parametrize("splits", [1, 3, 8])
def test_alu_kernel_splits(hb, splits):
    check(hb, case(27, "f32", 1, 18, 4, 2, 64, [700]), 20.0, True, num_splits=splits)
    check(hb, case(28, "f16", 1, 18, 4, 2, 128, [700]), 20.0, True, num_splits=splits)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("ps", [16, 64, 256])
@pytest.mark.parametrize("shape", [(2, 18, 4, 4, 128, [130, 0]), (2, 67, 16, 2, 128, [515, 90])], ids=["one_tile", "tile_pair"])
def test_paged_against_the_oracle(hb, dtype, ps, shape):
    c = case(29, dtype, *shape)
    q, k, v, lens, parent, slopes, pos = c
    B, Hkv, cap, D = k.shape
    per = -(-cap // ps)
    table = torch.randperm(B * per + 2, generator=torch.Generator().manual_seed(3))[:B * per].int().view(B, per).cuda()
    pools = []
    for t in (k, v):
        full = torch.full((B, Hkv, per * ps, D), float("nan"), dtype=t.dtype, device="cuda")
        full[:, :, :cap] = t
        pool = torch.full((B * per + 2, Hkv, ps, D), float("nan"), dtype=t.dtype, device="cuda")
        pool[table.long().flatten()] = full.view(B, Hkv, per, ps, D).permute(0, 2, 1, 3, 4).reshape(-1, Hkv, ps, D)
        pools.append(pool)
    for cap_s, bias in ((30.0, False), (0.0, True), (10.0, True)):
        out, st = hb.tree_attention_scored_paged(q, *pools, table, lens, parent, cap=cap_s, slopes=slopes if bias else None, pos=pos if bias else None)
        assert (st == 0).all()
        close(out, reference(c, cap_s, bias))


def test_bad_sequences_are_flagged_and_left_alone(hb):
    for dtype in ("f32", "bf16"):
        c = case(30, dtype, 4, 18, 4, 4, 128, [100, 90, 80, 70])
        q, k, v, lens, parent, slopes, pos = c
        lens[1] = -1
        lens[2] = k.shape[2] - 17
        parent[3, 5] = 5
        out = torch.full_like(q, 3.0)
        _, st = hb.tree_attention_scored(q, k, v, lens, parent, cap=30.0, slopes=slopes, pos=pos, out=out)
        assert st.tolist() == [0, 2, 2, 1]
        assert (out[1:] == 3).all()
        close(out[:1], [a[:1] for a in reference(c, 30.0, True)])


def test_captured_and_replayed_with_new_slopes_and_positions(hb):
    c = case(31, "bf16", 2, 18, 8, 8, 128, [300, 170])
    q, k, v, lens, parent, slopes, pos = c
    ws = torch.zeros(48 << 20, dtype=torch.uint8, device="cuda")
    hb.tree_attention_scored(q, k, v, lens, parent, cap=30.0, slopes=slopes, pos=pos, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(q)
    with torch.cuda.graph(graph, stream=side):
        slopes.mul_(0.5)                                                                # the kernel ahead writes what the call reads
        pos.add_(1)
        hb.tree_attention_scored(q, k, v, lens, parent, cap=30.0, slopes=slopes, pos=pos, workspace=ws, out=out,
                                 flags=hb.HT_ATTN_CONTEXT_FINAL)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        close(out, reference(c, 30.0, True))


def test_calls_on_two_streams_with_their_own_workspaces(hb):
    c1, c2 = case(32, "bf16", 2, 40, 8, 8, 128, [700, 900]), case(33, "bf16", 2, 67, 16, 2, 128, [700, 300])
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for c, s in zip((c1, c2), streams):
        with torch.cuda.stream(s):
            for _ in range(5):
                out, _ = hb.tree_attention_scored(*c[:5], cap=20.0, slopes=c[5], pos=c[6])
            outs.append(out)
    torch.cuda.synchronize()
    for c, out in zip((c1, c2), outs):
        close(out, reference(c, 20.0, True))


def test_binding_refuses_what_it_cannot_pass_on(hb):
    q, k, v, lens, parent, slopes, pos = case(34, "f16", 1, 4, 2, 2, 128, [8])
    with pytest.raises(ValueError):
        hb.tree_attention_scored(q, k, v, lens, parent, slopes=slopes)
    with pytest.raises(ValueError):
        hb.tree_attention_scored(q, k, v, lens, parent, slopes=slopes.double(), pos=pos)
    with pytest.raises(ValueError):
        hb.tree_attention_scored(q, k, v, lens, parent, slopes=slopes[:1], pos=pos)
    with pytest.raises(ValueError):
        hb.tree_attention_scored(q, k, v, lens, parent, slopes=slopes, pos=pos[:, :2])
    with pytest.raises(hb.HtError):
        hb.tree_attention_scored(q, k, v, lens, parent, cap=-1.0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(2, 18, 4, 4, 128, [130, 0]), (2, 91, 4, 4, 128, [1000, 64]), (1, 67, 16, 2, 128, [515])],
                         ids=lambda s: "N%dHq%dHkv%d" % s[1:4])
@pytest.mark.parametrize("away", [1000000, 70000, -1000000], ids=["far_behind", "behind", "far_ahead"])
def test_trees_placed_far_from_their_cache_rows(hb, dtype, shape, away):
    """Positions are given, and need not follow the cache rows: a cache that dropped rows has its tree far behind them, where
    only the tree's own keys weigh anything (positive slopes) and their distances are small differences of large positions.
    Far ahead (negative distances, a slope of 2^-20) every context key gains about as much."""
    q, k, v, lens, parent, slopes, pos = case(37, dtype, *shape)
    if away < 0:
        slopes = torch.full_like(slopes, 2.0 ** -20)      # the biases stay below two: their rounding is that of a score
    pos = pos + away
    check(hb, (q, k, v, lens, parent, slopes, pos), 0.0, True)
    check(hb, (q, k, v, lens, parent, slopes, pos), 20.0, True)


@pytest.mark.parametrize("q0", [87.0, 442.0, 1768.0, 17680.0])
def test_large_caps_shape_scores_on_either_side_of_half_of_them_alike(hb, q0):
    """One tile of scores a little above half the cap, one of scores a little below it: their forms must agree to the rounding
    of 32 bits.  Values of +1 and -1 weigh the two tiles against one another."""
    L, D = 256, 128
    cap = 2.0 * 64 * q0 / D ** 0.5                        # 64 products of q0 are half of it: 984 to 200026
    q, k, v = torch.zeros(1, 1, 1, D), torch.zeros(1, 1, L + 7, D), torch.ones(1, 1, L + 7, D)
    k[..., :64] = 1.0
    k[..., :128, 64], k[..., 128:, 64] = 0.002, -0.002
    v[..., 128:, :] = -1.0
    q[..., :65] = q0
    q, k, v = (t.half().cuda() for t in (q, k, v))
    lens, parent = torch.tensor([L], dtype=torch.int32, device="cuda"), torch.full((1, 1), -1, dtype=torch.int32, device="cuda")
    out, st = hb.tree_attention_scored(q, k, v, lens, parent, cap=cap)
    ref, size = so.tree_attention(f64(q), f64(k), f64(v), [L], parent.cpu().numpy(), cap, spread=True)
    # Beside the bound of `close`: the capped score of a tile is cap - 2 cap / (1 + e^(2t)) with the exponential off by 2^-22 and the
    # quotient by 2^-23 of themselves, which at t = 1/2 moves it by 2 * 0.27 * (0.73 * 2^-22 + 2^-23) = 1.6e-7 of the cap at most, or by
    # the rounding of its products, less than 0.4 * 2^-23 = 5e-8 of it; the difference of two scores moves the output by half as much.
    tol = 2.0 ** -11 * (size + np.abs(ref)) + 2e-5 * size + 2.0 ** -17 + 2.1e-7 * cap
    got = f64(out)
    assert (st == 0).all() and (np.abs(got - ref) <= tol).all(), (got[0, 0, 0, 0], ref[0, 0, 0, 0], tol[0, 0, 0, 0])


@pytest.mark.parametrize("shape", [(1, 18, 4, 4, 128, [40000]), (1, 67, 16, 2, 128, [36001])], ids=["one_tile", "tile_pair"])
@pytest.mark.parametrize("slope", [2.0 ** -13, 0.01], ids=["flat", "steep"])
def test_biased_rows_longer_than_two_to_the_fifteenth(hb, shape, slope):
    """A tile below 2^-40 of the reference is left out: of a part of n keys that is n 2^-40 of the weight at most, 2^-24 here."""
    c = case(38, "f16", *shape, slope=slope)
    check(hb, c, 0.0, True)
    check(hb, c, 20.0, True)


@pytest.mark.parametrize("ps", [16, 256])
@pytest.mark.parametrize("shape", [(2, 18, 4, 4, 128, [900, 0]), (2, 67, 16, 2, 128, [1300, 90]), (5, 19, 16, 16, 128, [600, 20, 900, 333, 128])],
                         ids=["few", "tile_pair", "many_units"])
def test_paged_with_the_two_promises(hb, ps, shape):
    """A kept workspace whose counters reset themselves, and context rows that are final ahead of the call."""
    c = case(39, "bf16", *shape)
    q, k, v, lens, parent, slopes, pos = c
    B, Hkv, cap, D = k.shape
    per = -(-cap // ps)
    table = torch.randperm(B * per + 2, generator=torch.Generator().manual_seed(4))[:B * per].int().view(B, per).cuda()
    pools = []
    for t in (k, v):
        full = torch.full((B, Hkv, per * ps, D), float("nan"), dtype=t.dtype, device="cuda")
        full[:, :, :cap] = t
        pool = torch.full((B * per + 2, Hkv, ps, D), float("nan"), dtype=t.dtype, device="cuda")
        pool[table.long().flatten()] = full.view(B, Hkv, per, ps, D).permute(0, 2, 1, 3, 4).reshape(-1, Hkv, ps, D)
        pools.append(pool)
    ws = torch.zeros(48 << 20, dtype=torch.uint8, device="cuda")
    for cap_s, bias in ((30.0, False), (0.0, True), (10.0, True)):
        ref = reference(c, cap_s, bias)
        for _ in range(3):
            out, st = hb.tree_attention_scored_paged(q, *pools, table, lens, parent, cap=cap_s, slopes=slopes if bias else None,
                                                     pos=pos if bias else None, workspace=ws,
                                                     flags=hb.HT_ATTN_WORKSPACE_CLEAN | hb.HT_ATTN_CONTEXT_FINAL)
            assert (st == 0).all()
            close(out, ref)


@pytest.mark.parametrize("shape", [(3, 18, 4, 4, 128, [130, 200, 90]), (3, 67, 16, 2, 128, [515, 300, 90])], ids=["one_tile", "tile_pair"])
def test_paged_bad_pages_and_lengths_are_flagged_alone(hb, shape):
    c = case(40, "bf16", *shape)
    q, k, v, lens, parent, slopes, pos = c
    B, Hkv, cap, D = k.shape
    ps = 16
    per = -(-cap // ps)
    table = torch.arange(B * per, dtype=torch.int32, device="cuda").view(B, per).contiguous()
    pools = []
    for t in (k, v):
        full = torch.zeros((B, Hkv, per * ps, D), dtype=t.dtype, device="cuda")
        full[:, :, :cap] = t
        pools.append(full.view(B, Hkv, per, ps, D).permute(0, 2, 1, 3, 4).reshape(-1, Hkv, ps, D).contiguous())
    for kw in (dict(cap=10.0), dict(slopes=slopes, pos=pos), dict(cap=10.0, slopes=slopes, pos=pos)):
        ref = reference(c, kw.get("cap", 0.0), "slopes" in kw)
        for page in (-1, B * per, 2 ** 30):
            bad = table.clone()
            bad[1, 3] = page
            bad[2, -1] = page                                  # behind the sequence's last row: not needed
            out, st = hb.tree_attention_scored_paged(q, *pools, bad, lens, parent, **kw)
            assert st.tolist() == [0, hb.HT_STATUS_BAD_PAGE, 0]
            close(out[::2], [a[::2] for a in ref])
        wrong = lens.clone()
        wrong[0] = per * ps
        out, st = hb.tree_attention_scored_paged(q, *pools, table, wrong, parent, **kw)
        assert st.tolist() == [2, 0, 0]
        close(out[1:], [a[1:] for a in ref])
