"""Sampling and sampled verification on the GPU against the fp64 oracle: tokens are whole numbers and have to be equal."""
import math

import numpy as np
import pytest
import torch

from oracle import sample_oracle as so

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def hb():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2404_12022_b200 import binding
    binding.load()
    return binding


def dev(a, t=torch.float32):
    return None if a is None else torch.as_tensor(np.asarray(a), dtype=t).cuda()


def check(hb, x, u, T=None, k=None, p=None, m=None, what=""):
    """x [B, N, V] CUDA logits, u [B, N]."""
    got, st = hb.sample(x, dev(u), dev(T), dev(k, torch.int32), dev(p), dev(m))
    f = lambda a: None if a is None else np.asarray(a, np.float32).astype(np.float64)   # noqa: E731
    want = so.sample(x.double().cpu().numpy(), f(u), f(T), k, f(p), f(m))
    assert (st == 0).all()
    assert np.array_equal(got.cpu().numpy(), want), "%s: %s" % (what, np.argwhere(got.cpu().numpy() != want)[:5])


def logits(seed, dt, B, N, V, spread=2.0, boost=8.0):
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn((B, N, V), generator=g)
    at = torch.randint(0, V, (B, N, 1), generator=g)
    x.scatter_add_(2, at, boost * torch.rand((B, N, 1), generator=g))
    return x.to(dt).cuda(), torch.rand((B, N), generator=g).numpy()


FILTERS = [dict(), dict(T=0.7), dict(k=1), dict(k=2), dict(k=50), dict(k=600), dict(p=0.1), dict(p=0.5), dict(p=0.95), dict(p=0.999),
           dict(m=0.05), dict(k=40, p=0.9), dict(k=700, p=0.9), dict(k=700, p=0.97, m=0.01, T=1.3), dict(p=0.8, m=0.1), dict(T=0.05),
           dict(T=0.05, k=100), dict(T=0.02, k=600, p=0.9), dict(T=20.0, p=0.6), dict(T=0.0, p=0.3)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 1000, 5003])
@pytest.mark.parametrize("kw", FILTERS, ids=lambda k: "_".join("%s%g" % i for i in k.items()) or "none")
def test_tokens_are_those_of_the_oracle(hb, dtype, V, kw):
    B, N = 3, 4
    x, u = logits(41, DT[dtype], B, N, V)
    check(hb, x, u, **{n: [v] * B for n, v in kw.items()}, what=str(kw))


@pytest.mark.parametrize("dtype,V", [("bf16", 32000), ("f32", 70001), ("f16", 120007), ("bf16", 200001)])
@pytest.mark.parametrize("spread", [0.5, 2.5])
def test_large_vocabularies_each_sequence_with_its_own_parameters(hb, dtype, V, spread):
    """Rows in shared memory and rows too long for it, flat and peaked, long nuclei and short ones."""
    x, u = logits(42, DT[dtype], 6, 1, V, spread, 6 * spread)
    check(hb, x, u, T=[1.0, 0.6, 1.4, 0.0, 0.8, 1.0], k=[0, 50, 3000, 5, -1, V], p=[0.9, 0.95, 0.99, 1.0, 1.5, 0.3], m=[0.0, 0.0, 0.01, 0.5, 0.001, -1.0])


def test_uniform_numbers_at_the_ends(hb):
    x, _ = logits(43, torch.float32, 2, 3, 400, 3.0)
    u = np.array([[0.0, 1.0, np.nextafter(np.float32(1), np.float32(0))]] * 2, np.float32)
    for kw in (dict(), dict(k=[5, 5]), dict(p=[0.9, 0.9]), dict(m=[0.2, 0.2]), dict(T=[0.01, 0.01]), dict(k=[600, 390], p=[0.99, 0.99])):
        check(hb, x, u, **kw)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V,N", [(30, 2000), (500, 500), (5003, 100), (60001, 8)])
@pytest.mark.parametrize("kw", [dict(), dict(k=20), dict(k=700), dict(T=2.0)], ids=str)
def test_uniform_one_takes_the_last_kept_token_with_a_weight(hb, dtype, V, N, kw):
    """Tokens whose weight is lost in the rounding of the sum count as well: no running weight exceeds all of it."""
    x, _ = logits(57, DT[dtype], 1, N, V, spread=12.0)
    got, st = hb.sample(x, torch.ones((1, N), device="cuda"), dev([kw["T"]]) if "T" in kw else None, dev([kw["k"]], torch.int32) if "k" in kw else None)
    a = x[0].double().cpu().numpy()
    order = np.argsort(-a, axis=1, kind="stable")[:, :kw.get("k", V)]
    assert ((a.max(1) - a.min(1)) < 600).all()                                          # every weight is above 2^-1000
    assert (st == 0).all() and np.array_equal(got[0].cpu().numpy(), order.max(1))


def test_weights_far_below_the_largest_still_count(hb):
    """With uniform 0 the first token of any weight is the answer, down to 2^-1000 of the largest and not below."""
    x = torch.full((3, 1, 900), -float("inf"))
    x[:, 0, 700] = 0.0
    x[0, 0, 3], x[1, 0, 3], x[2, 0, 3] = -500.0, -690.0, -700.0
    x = x.cuda()
    check(hb, x, np.zeros((3, 1)))
    got, _ = hb.sample(x, torch.zeros((3, 1), device="cuda"))
    assert got.flatten().tolist() == [3, 3, 700]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [6, 3000, 40003])
def test_rows_of_equal_logits_and_of_few_values(hb, dtype, V):
    """Ties far beyond what the list of candidates holds: the cut runs through equal tokens, by index."""
    B = 8
    x = torch.zeros((B, 2, V))
    g = torch.Generator().manual_seed(4)
    x[:, 1] = torch.randint(-2, 2, (B, V), generator=g).float()
    x[4:, 0] = -3.5
    u = torch.rand((B, 2), generator=g).numpy()
    check(hb, x.to(DT[dtype]).cuda(), u, p=[0.5, 0.9, 0.25, 1.0] * 2, k=[0, 0, 2000, 1500, 5, 700, 0, 0])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_nan_infinities_masks_and_signed_zeros(hb, dtype):
    dt, V, inf, nan = DT[dtype], 1500, float("inf"), float("nan")
    g = torch.Generator().manual_seed(9)
    x = torch.randn((12, 1, V), generator=g)
    x[0] = nan
    x[1] = -inf
    x[2, 0] = nan
    x[2, 0, 40:] = -inf
    x[3, 0, ::3] = nan
    x[4, 0, ::2] = -inf
    x[5, 0, 100], x[5, 0, 900] = inf, inf
    x[6, 0, 5:] = torch.finfo(dt).min                                                   # a mask of the type's lowest value
    x[7] = torch.finfo(dt).min
    x[8, 0] = 0.0
    x[8, 0, ::2] = -0.0
    x[9, 0, 1:] = -inf
    x[10, 0, 100], x[10, 0, 3], x[10, 0, 4] = inf, nan, -inf
    x = x.to(dt).cuda()
    for seed in range(4):
        u = np.random.default_rng(seed).random((12, 1)).astype(np.float32)
        for kw in (dict(), dict(k=[600] * 12), dict(k=[3] * 12), dict(p=[0.7] * 12), dict(T=[0.0] * 12), dict(m=[0.3] * 12), dict(k=[20] * 12, p=[0.9] * 12)):
            check(hb, x, u, **kw, what=str(kw))


def test_cuts_among_tokens_far_below_the_largest(hb):
    """The k-th token, or the end of a nucleus of 1 - 1e-7, lies below 2^-32 of the largest weight."""
    g = torch.Generator().manual_seed(12)
    x = torch.randn((6, 1, 4000), generator=g)
    x[:, 0, 17] = 60.0
    u = np.array([[0.5], [1.0], [0.9999999], [0.3], [1.0], [0.99999994]], np.float32)
    check(hb, x.cuda(), u, k=[700, 700, 2000, 0, 0, 0], p=[1.0, 0.9, 1.0, 0.9999999, 0.99999994, 0.9999])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [4000, 22318, 131072])
def test_cuts_by_count_far_below_the_largest(hb, dtype, V):
    """The k-th token far below the largest, among values that are all distinct (where the type has them), among ties that
    the list of candidates holds and among ties that it does not, with masked tokens between; u = 1 takes the last kept one."""
    g = torch.Generator().manual_seed(77)
    x = torch.randn((6, 1, V), generator=g)
    x[2] = (20 * x[2]).round() / 20
    x[3] = x[3].round()
    x[4, 0, ::3] = float("-inf")
    x[5, 0, ::3] = torch.finfo(DT[dtype]).min
    x[:, 0, V // 2] = 70.0
    u = np.array([[1.0], [0.5], [1.0], [1.0], [1.0], [1.0]], np.float32)
    for k in (513, 1789, V // 2, V - 1):
        check(hb, x.to(DT[dtype]).cuda(), u, k=[k] * 6, p=[1.0] * 5 + [0.99999994], what=str(k))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [1200, 6007, 60001])
def test_nuclei_that_hold_all_of_a_top_k_cut_through_ties(hb, dtype, V):
    """top_k ends among equal tokens and top_p is so near 1 that nothing else is cut: the tokens equal to the k-th, but
    behind it, stay out.  (The k-th token carries at least 1e-6 of the weight, so top_p of 1 - 6e-8 to 1 - 1e-7 ends behind it.)"""
    g = torch.Generator().manual_seed(31)
    x = torch.randint(0, 8, (8, 1, V), generator=g).float() / 8                       # 150 to 7500 tokens of each value
    x[4:] = torch.randint(0, 40, (4, 1, V), generator=g).float() / 40
    x[3], x[7] = 0.0, 1.5                                                             # one value throughout
    x = x.to(DT[dtype]).cuda()
    for u in (0.0, 0.31, 0.77, 0.999):
        for k in (3, 100, 300, 513, 700, 1100):
            for p in (0.9999999, 0.99999994):
                check(hb, x, np.full((8, 1), u, np.float32), k=[k] * 8, p=[p] * 8, what=str((u, k, p)))
                check(hb, x, np.full((8, 1), u, np.float32), k=[k] * 8, p=[p] * 8, m=[0.5, 0.0] * 4, what=str((u, k, p, "min_p")))


@pytest.mark.parametrize("V", [700, 9001, 40003])
def test_bf16_nuclei_wherever_the_cut_lies(hb, V):
    """The cut among positive, negative and equal values, among values next to zero, in rows far from zero, in rows whose
    smaller values lie beyond the counted range; rows over one block and over several."""
    g = torch.Generator().manual_seed(61)
    rnd = torch.randn((10, 1, V), generator=g)
    x = torch.stack([rnd[0], rnd[1] * 1e-3, rnd[2] * 1e-6 + 0.0, rnd[3] * 3 - 40.0, rnd[4] * 60.0 - 300.0, rnd[5] * 3 + 180.0,
                     (rnd[6] * 2).round(), rnd[7].clamp(max=0.0), -rnd[8].abs() * 20.0, rnd[9] * 0.01 + 1.0])
    x = x.to(torch.bfloat16).cuda()
    for seed, p in enumerate((0.2, 0.5, 0.62, 0.9, 0.999)):
        u = np.random.default_rng(seed).random((10, 1)).astype(np.float32)
        for T in (1.0, 0.3, 30.0):
            check(hb, x, u, T=[T] * 10, p=[p] * 10, what="p %g T %g" % (p, T))
        check(hb, x, u, p=[p] * 10, m=[0.3] * 10, what="p %g and min_p" % p)
        check(hb, x, np.zeros((10, 1)), p=[p] * 10, what="p %g, uniform 0" % p)


def test_a_row_too_long_for_shared_memory(hb):
    x, u = logits(62, torch.float32, 2, 1, 500001, 2.0, 10.0)
    check(hb, x, u)
    check(hb, x, u, k=[40, 900], p=[0.9, 0.95])
    check(hb, x, u, p=[0.3, 0.9])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_extreme_parameters(hb, dtype):
    V = 2000
    x, u = logits(63, DT[dtype], 8, 2, V)
    check(hb, x, u, T=[1e-30, 1e-38, 1e-3, 1e3, 1e10, 1e30, 1.0, 1.0])
    check(hb, x, u, T=[1e-30, 1e-3, 1e3, 1e10] * 2, p=[0.5] * 8)
    check(hb, x, u, k=[V - 1, V, V + 1, 2 ** 31 - 1, -(2 ** 31), 512, 513, 1])
    check(hb, x, u, p=[1e-30, 1e-6, 0.9999999, 1.0, 2.0, 0.0, -1.0, 1.0], m=[0, 0, 0, 1.0, 0.999, 1e-30, 0.5, -3.0])


def test_bad_parameters_are_flagged(hb):
    B, nan, inf = 9, float("nan"), float("inf")
    x, _ = logits(44, torch.float16, B, 2, 300)
    u = np.full((B, 2), 0.4, np.float32)
    u[6, 1], u[7, 0], u[8, 1] = -0.1, 1.5, nan
    T = np.array([1, -1, inf, nan, 1, 1, 1, 1, 1], np.float32)
    p, m = np.full(B, 0.9, np.float32), np.zeros(B, np.float32)
    p[4], m[5] = nan, 1.5
    got, st = hb.sample(x, dev(u), dev(T), None, dev(p), dev(m))
    assert st.tolist() == [0] + [hb.HT_STATUS_BAD_PARAM] * 8
    assert (got[1:] == -1).all() and (got[0] >= 0).all()


def test_frequencies_over_many_uniform_numbers(hb):
    """20000 draws from one row: each frequency within five standard deviations of its probability (inputs fixed)."""
    n, V = 20000, 16
    x = torch.randn(V, generator=torch.Generator().manual_seed(2))
    u = (torch.arange(n, dtype=torch.float32) + 0.5) / n                                 # evenly spread: counts within one of n p
    got, _ = hb.sample(x.expand(1, n, V).contiguous().cuda(), u[None].cuda())
    p = torch.softmax(x.double(), 0)
    assert ((torch.bincount(got.flatten().cpu(), minlength=V) - n * p).abs() <= 1.01).all()


# ---------------------------------------------------------------------------------------------------------------------
def trees(rng, B, T, N):
    parent = np.full((B, N), -1, np.int32)
    for b in range(B):
        for r in range(1, N):
            parent[b, r] = rng.integers(max(-1, r - 6), r)
    return parent


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 50), (2, 15, 18, 64), (3, 88, 91, 300), (2, 300, 300, 40), (2, 20, 23, 32003)],
                         ids=lambda s: "B%dT%dN%dV%d" % s)
@pytest.mark.parametrize("root", [True, False])
def test_sampled_verification_is_sampling_and_the_path_search(hb, oracle, dtype, shape, root):
    B, T, N, V = shape
    rng = np.random.default_rng(7)
    x, u = logits(45, DT[dtype], B, N, V, 2.0, 20.0)
    parent = trees(rng, B, T, N)
    f64 = lambda a: np.asarray(a, np.float32).astype(np.float64)                        # noqa: E731
    Tm, k, p = [0.9] * B, [30] * B, [0.9] * B
    pred = np.full((B, N), -1, np.int32)
    pred[:, :T] = so.sample(x.double().cpu().numpy()[:, :T], f64(u), f64(Tm), k, f64(p))
    # drafts that follow the samples with probability 0.7, so that paths of several nodes are accepted
    root_pred = rng.integers(0, V, B).astype(np.int32)
    tokens = rng.integers(0, V, (B, T)).astype(np.int32)
    for b in range(B):
        for c in range(T):
            if rng.random() < 0.7:
                tokens[b, c] = root_pred[b] if parent[b, c] < 0 else pred[b, parent[b, c]]
    accept_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    for _ in range(2):                                                                  # the second call starts from the first one's lengths
        got = hb.verify_sampled(x, dev(u), dev(tokens, torch.int32), dev(parent, torch.int32), dev(root_pred, torch.int32) if root else None,
                                dev(Tm), dev(k, torch.int32), dev(p), max_path=64, accept_len=accept_len)
        want = oracle.accept_scan(tokens, parent, pred, root_pred if root else None, 64)
        assert np.array_equal(got[0].cpu().numpy(), pred)
        for g, w, name in zip(got[1:], want, ("accept_len", "accept_path", "next_token", "status")):
            assert np.array_equal(g.cpu().numpy(), w), name


def test_greedy_temperature_is_the_greedy_verification(hb):
    B, T, N, V = 3, 60, 64, 5000
    x, u = logits(46, torch.bfloat16, B, N, V)
    parent = dev(trees(np.random.default_rng(3), B, T, N), torch.int32)
    greedy = x.float().argmax(-1).int()
    tokens = torch.gather(greedy, 1, parent[:, :T].clamp(min=0).long()).contiguous()
    a = hb.verify_greedy(x, tokens, parent, greedy[:, 0].contiguous(), 64)
    b = hb.verify_sampled(x, dev(u), tokens, parent, greedy[:, 0].contiguous(), temperature=torch.zeros(B, device="cuda"), max_path=64)
    assert torch.equal(a[0][:, :T], b[0][:, :T]) and all(torch.equal(p, q) for p, q in zip(a[1:], b[1:]))


def test_statuses_of_sampled_verification(hb):
    B, T, V = 4, 12, 100
    x, u = logits(47, torch.float32, B, T, V)
    parent = np.tile(np.arange(-1, T - 1, dtype=np.int32), (B, 1))                       # chains
    parent[1, 4] = 4
    u[2, 7] = 2.0
    pred = hb.sample(x, dev(np.clip(u, 0, 1)))[0]
    tokens = torch.cat((torch.zeros((B, 1), dtype=torch.int32, device="cuda"), pred[:, :-1]), 1).contiguous()
    got = hb.verify_sampled(x, dev(u), tokens, dev(parent, torch.int32), None, max_path=5)
    assert got[4].tolist() == [4, 1, hb.HT_STATUS_BAD_PARAM, 4]
    assert got[1].tolist() == [0] * 4 and got[3].tolist() == [-1] * 4 and (got[0][2] == -1).all() and (got[2][2] == -1).all()
    u[2, 7] = 0.5
    got = hb.verify_sampled(x, dev(u), tokens, dev(parent, torch.int32), None, max_path=12, accept_len=got[1])
    assert got[4].tolist() == [0, 1, 0, 0] and got[1].tolist()[0] == T


def test_more_rows_than_the_tree_search_stages(hb, oracle):
    B, N, V = 2, 1100, 40
    x, u = logits(49, torch.bfloat16, B, N, V, 2.0, 20.0)
    parent = trees(np.random.default_rng(4), B, N, N)
    pred = so.sample(x.double().cpu().numpy(), u.astype(np.float64))
    tokens = np.take_along_axis(pred, np.maximum(parent, 0), 1)
    got = hb.verify_sampled(x, dev(u), dev(tokens, torch.int32), dev(parent, torch.int32), None, max_path=255)
    want = oracle.accept_scan(tokens, parent, pred, None, 255)
    for g, w in zip(got, (pred, *want)):
        assert np.array_equal(g.cpu().numpy(), w)


def test_captured_and_replayed_and_two_streams(hb, oracle):
    B, T, V = 2, 40, 4000
    sets = [logits(s, torch.bfloat16, B, T, V, 2.0, 15.0) for s in (50, 51, 52)]
    x, u = sets[0][0].clone(), dev(sets[0][1])
    parent = dev(trees(np.random.default_rng(1), B, T, T), torch.int32)
    tokens = torch.randint(0, V, (B, T), generator=torch.Generator().manual_seed(0)).int().cuda()
    p = torch.full((B,), 0.9, device="cuda")
    alen = torch.zeros(B, dtype=torch.int32, device="cuda")
    hb.verify_sampled(x, u, tokens, parent, None, top_p=p, accept_len=alen)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = hb.verify_sampled(x, u, tokens, parent, None, top_p=p, accept_len=alen)
    for xs, us in sets[1:]:
        x.copy_(xs)
        u.copy_(dev(us))
        graph.replay()
        torch.cuda.synchronize()
        want = so.sample(xs.double().cpu().numpy(), us.astype(np.float64), None, None, np.full(B, np.float32(0.9), np.float64))
        assert np.array_equal(out[0].cpu().numpy(), want)
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for (xs, us), s in zip(sets[1:], streams):
        with torch.cuda.stream(s):
            got.append(hb.sample(xs, dev(us), top_p=p)[0])
    torch.cuda.synchronize()
    for (xs, us), t in zip(sets[1:], got):
        assert np.array_equal(t.cpu().numpy(), so.sample(xs.double().cpu().numpy(), us.astype(np.float64), None, None,
                                                         np.full(B, np.float32(0.9), np.float64)))


def test_binding_refuses_what_it_cannot_pass_on(hb):
    x, u = logits(48, torch.float16, 2, 3, 50)
    for kw in (dict(u=dev(u)[:1]), dict(u=dev(u).double()), dict(T=torch.ones(3, device="cuda")), dict(k=torch.ones(2, device="cuda")), dict(T=torch.ones(2))):
        with pytest.raises(ValueError):
            hb.sample(x, kw.get("u", dev(u)), kw.get("T"), kw.get("k"))


@pytest.mark.parametrize("V,gap", [(1 << 24, 22.22), (1 << 24, 22.7), (1 << 25, 22.5), (1 << 25, 22.67)])
def test_nuclei_that_end_in_a_far_tail_of_very_many_equal_tokens(hb, V, gap):
    """One token, and V - 1 equal ones below 2^-32 of it that together weigh as much as 0.2 to 0.8 % of it; the nucleus leaves
    2^-24 of the whole out.  Where the whole is a 32-bit sum, its rounding is more than that: no token would end the nucleus.
    The last kept token (uniform = 1) is known in closed form."""
    x = torch.full((1, 1, V), -gap, device="cuda")
    x[0, 0, V // 2] = 0.0
    p = 1.0 - 2.0 ** -24
    w = math.exp(float(x[0, 0, 0]))
    n = (p * (1.0 + (V - 1) * w) - 1.0) / w              # equal tokens before which less than the goal has come: this rounded up
    assert 0.05 < n % 1 < 0.95                           # (the kernel's weights are good to 1e-12: 0.01 of a token here)
    last = math.ceil(n) - 1                              # as the index among the equal tokens
    got, st = hb.sample(x, dev([[1.0]]), None, None, dev([p]))
    assert st.tolist() == [0] and got.item() == last + (last >= V // 2), (got.item(), last)
    assert hb.sample(x, dev([[0.5]]), None, None, dev([p]))[0].item() == V // 2


@pytest.mark.parametrize("kw", [dict(), dict(p=0.9999), dict(k=1 << 20, p=0.99995), dict(k=(1 << 20) + 7)], ids=lambda k: "_".join(k) or "none")
@pytest.mark.parametrize("dtype,V,gap", [("f32", 1 << 24, 22.31), ("f16", (1 << 23) + 1, 22.0), ("bf16", (1 << 21) + 3, 21.625)])
def test_draws_from_a_far_tail_of_very_many_equal_tokens(hb, dtype, V, gap, kw):
    """As above: the token that a uniform number meets within the tail is known in closed form, and a 32-bit sum of the tail
    would move it by some tens of tokens or more."""
    x = torch.full((1, 1, V), -gap, device="cuda").to(DT[dtype])
    x[0, 0, 0] = 0.0
    w = math.exp(float(x[0, 0, 1]))
    n = min(kw.get("k", V), V) - 1                       # equal tokens kept
    if "p" in kw:
        p = float(np.float32(kw["p"]))
        n_p = (p * (1.0 + n * w) - 1.0) / w
        assert 0.01 < n_p % 1 < 0.99
        n = math.ceil(n_p)
    whole = 1.0 + n * w
    for f in (0.1, 0.5, 0.93):                            # how far into the tail
        u = float(np.float32((1.0 + f * n * w) / whole))
        at = (u * whole - 1.0) / w                       # tokens passed when the goal is met
        while not 0.05 < at % 1 < 0.95:                  # (the kernel's sums are good to 0.01 of a token)
            u = float(np.nextafter(np.float32(u), np.float32(0)))
            at = (u * whole - 1.0) / w
        got, st = hb.sample(x, dev([[u]]), None, dev([kw["k"]], torch.int32) if "k" in kw else None, dev([kw["p"]]) if "p" in kw else None)
        assert st.tolist() == [0] and got.item() == math.floor(at) + 1, (f, got.item(), at)


@pytest.mark.parametrize("N", [2048, 2049, 5000])
def test_many_rows_and_their_bad_numbers(hb, oracle, N):
    """Sequences of more rows than every block looks through itself: flagged all the same, by any parameter and by a uniform
    number anywhere, and only they."""
    B, V = 6, 24
    x, u = logits(43, torch.float32, B, N, V)
    u[1, N - 1], u[2, 0], u[3, N // 2] = 1.5, -1e-9, np.nan
    T, p = np.full(B, 0.8, np.float32), np.full(B, 0.9, np.float32)
    T[4] = -1.0
    want = so.sample(x.double().cpu().numpy(), u.astype(np.float64), np.where(T < 0, 1, T).astype(np.float64), None, p.astype(np.float64))
    want[1:5] = -1
    for _ in range(2):
        got, st = hb.sample(x, dev(u), dev(T), None, dev(p))
        assert st.tolist() == [0, 7, 7, 7, 7, 0] and np.array_equal(got.cpu().numpy(), want)
    # the verification looks at the rows of the tree alone
    rows = N - 1
    rng = np.random.default_rng(44)
    tokens, parent = rng.integers(0, V, (B, rows)).astype(np.int32), trees(rng, B, rows, N)
    pred, alen, path, nxt, st = hb.verify_sampled(x, dev(u), dev(tokens, torch.int32), dev(parent, torch.int32), None, dev(T), None, dev(p))
    assert st.tolist() == [0, 0, 7, 7, 7, 0] and (pred[2:5] == -1).all() and alen[2:5].tolist() == [0, 0, 0] and nxt[2:5].tolist() == [-1] * 3
    full = np.full((B, N), -1, np.int32)
    u[1, N - 1] = 0.5
    full[:, :rows] = so.sample(x.double().cpu().numpy(), u.astype(np.float64), np.where(T < 0, 1, T).astype(np.float64), None, p.astype(np.float64))[:, :rows]
    good = [0, 1, 5]
    ref = oracle.accept_scan(tokens[good], parent[good], full[good], None, 8)
    for g, w in zip((pred, alen, path, nxt, st), (full[good], *ref)):
        assert np.array_equal(g.cpu().numpy()[good], w)
