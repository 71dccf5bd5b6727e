"""Shaped logits and token counts on the GPU against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as qo

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def hb():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2404_12022_b200 import binding
    binding.load()
    return binding


def host(t):
    return None if t is None else t.cpu().numpy()


def close(got, want, terms):
    """One rounding to the type, half a step (float16: of its smallest, 2^-25, at least); before it at most eight roundings of 32 bits
    on values no larger than `terms`, the sum of what is added up."""
    g = got.double().cpu().numpy()
    fine = np.isfinite(want)
    assert np.array_equal(g[~fine], want[~fine], equal_nan=True)
    tol = torch.finfo(got.dtype).eps / 2 * np.abs(want[fine]) + 8 * 2.0 ** -24 * terms + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
    assert (np.abs(g[fine] - want[fine]) <= tol).all(), np.abs(g[fine] - want[fine]).max()


class Case:
    def __init__(self, seed, dtype, B, T, pseudo, V, seen=20, n_bias=0, masked=False, twice=False, chain=False):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        N = T + pseudo
        self.x = (2.5 * torch.randn((B, N, V), generator=g)).to(DT[dtype]).cuda()
        counts = torch.zeros((B, V), dtype=torch.int32)
        for b in range(B):
            for v in rng.integers(0, V, seen):
                counts[b, v] += 2 if rng.random() < 0.7 else 0
                counts[b, v] |= int(rng.random() < 0.3)
        parent = np.full((B, N), -1, np.int32)
        for b in range(B):
            for r in range(1, N):
                parent[b, r] = r - 1 if chain else rng.integers(max(-1, r - 5), r)
        few = rng.integers(0, V, 3)                                                     # drafts that repeat
        tokens = np.where(rng.random((B, T)) < 0.5, rng.choice(few, (B, T)), rng.integers(0, V, (B, T))).astype(np.int32)
        col = lambda lo, hi: (torch.rand(B, generator=g) * (hi - lo) + lo).cuda()       # noqa: E731
        self.kw = dict(counts=counts.cuda(), tokens=torch.from_numpy(tokens).cuda(), parent=torch.from_numpy(parent).cuda(), repetition=col(0.8, 1.5),
                       frequency=col(-0.5, 0.9), presence=col(-0.5, 0.9))
        if n_bias:
            ids = rng.integers(-2, V + 2, (B, n_bias)) if twice else np.stack([rng.permutation(V)[:n_bias] for _ in range(B)])
            self.kw.update(bias_id=torch.from_numpy(ids.astype(np.int32)).cuda(), bias=(4 * torch.randn((B, n_bias), generator=g)).cuda())
        if masked:
            words = rng.integers(-2 ** 31, 2 ** 31, (B, N, (V + 31) // 32)).astype(np.int32)
            words[0, 0] = 0                                                             # nothing is allowed
            words[0, N - 1] = -1
            self.kw["allowed"] = torch.from_numpy(words).cuda()

    def check(self, hb, in_place=False, **change):
        kw = dict(self.kw, **change)
        x = self.x.clone()
        out, st = hb.shape_logits(x, out=x if in_place else None, **kw)
        want, status = qo.shape_logits(self.x.double().cpu().numpy(), **{k: host(v) for k, v in kw.items()})
        assert st.tolist() == status.tolist() == [0] * len(status)
        terms = 30.0 + (0.0 if kw.get("bias") is None else float(kw["bias"].abs().sum(1).max()) if kw["bias"].shape[1] > 40 else 200.0)
        count = 0.0 if kw.get("counts") is None else float(kw["counts"].max())
        close(out, want, terms + count + len(want[0]))
        if not in_place:
            assert torch.equal(x.view(torch.uint8), self.x.view(torch.uint8))
        return out


SHAPES = [(1, 1, 0, 5), (2, 5, 2, 33), (1, 88, 3, 4096), (3, 7, 1, 4097), (2, 20, 3, 12001), (2, 40, 0, 8191), (1, 3, 1, 32000)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%dx%d+%d_%d" % s)
@pytest.mark.parametrize("in_place", [False, True], ids=["apart", "in_place"])
def test_everything_together(hb, dtype, shape, in_place):
    B, T, P, V = shape
    c = Case(sum(shape), dtype, *shape, seen=min(V, 300), n_bias=min(V, 60), masked=True)
    c.check(hb, in_place)
    c.check(hb, in_place, allowed=None)
    c.check(hb, in_place, bias_id=None, bias=None)
    c.check(hb, in_place, counts=None)
    c.check(hb, in_place, tokens=None, parent=None)
    c.check(hb, in_place, repetition=None, frequency=None, presence=None)


def test_nothing_to_shape_is_a_copy(hb):
    c = Case(1, "bf16", 2, 4, 1, 999)
    out, st = hb.shape_logits(c.x)
    assert torch.equal(out, c.x) and st.tolist() == [0, 0]


def test_biases_of_one_token_add_up(hb):
    for n in (2, 300, 1024):
        Case(n, "f32", 3, 6, 0, 200, n_bias=n, twice=True).check(hb)
    x = torch.zeros((1, 1, 40), device="cuda")
    ids = torch.tensor([[7, 7, 7, 3, -1, 40]], dtype=torch.int32, device="cuda")
    out, _ = hb.shape_logits(x, bias_id=ids, bias=torch.tensor([[0.0, 2.0, 0.0, -float("inf"), 9.0, 9.0]], device="cuda"))
    assert out[0, 0, 7] == 2 and out[0, 0, 3] == -float("inf") and out.nan_to_num(neginf=0).sum() == 2


def test_a_long_path_of_one_token(hb):
    """1024 rows, a chain; all draft tokens alike: row r has seen it r + 1 times."""
    c = Case(3, "f32", 1, 1024, 0, 50, seen=0, chain=True)
    c.kw["tokens"].fill_(11)
    out = c.check(hb)
    gap = (c.x - out)[0, :, 11]
    assert (gap[1000] - gap[10]).item() > 100 * abs(float(c.kw["frequency"][0])) or float(c.kw["frequency"][0]) < 0.2


def test_values_that_are_no_numbers(hb):
    c = Case(4, "f16", 1, 3, 0, 700, seen=400, n_bias=30, masked=True)
    c.x[0, 1, ::5] = float("nan")
    c.x[0, 1, 1::5] = float("inf")
    c.x[0, 2, 2::5] = -float("inf")
    c.check(hb)
    c.check(hb, in_place=True)


def test_statuses_leave_rows_alone(hb):
    for name, bad in (("repetition", 0.0), ("repetition", float("nan")), ("repetition", float("inf")), ("frequency", float("inf")), ("presence", float("nan"))):
        c = Case(5, "bf16", 3, 4, 1, 5000, masked=True)
        c.kw[name][1] = bad
        out = torch.full_like(c.x, 3.0)
        _, st = hb.shape_logits(c.x, out=out, **c.kw)
        assert st.tolist() == [0, 7, 0] and (out[1] == 3.0).all()
        want, _ = qo.shape_logits(c.x.double().cpu().numpy(), **{k: host(v) for k, v in c.kw.items()})
        close(out[[0, 2]], want[[0, 2]], 80.0)
    c = Case(6, "bf16", 2, 4, 1, 300)
    c.kw["parent"][1, 4] = 4
    out = torch.full_like(c.x, 3.0)
    assert hb.shape_logits(c.x, out=out, **c.kw)[1].tolist() == [0, 1] and (out[1] == 3.0).all()


def test_drafts_outside_the_vocabulary_touch_nothing(hb):
    c = Case(7, "f32", 1, 6, 0, 100)
    c.kw["tokens"][0, 1], c.kw["tokens"][0, 2] = -1, 100
    c.check(hb)


@pytest.mark.parametrize("B,n,V", [(1, 1, 1), (3, 40, 17), (2, 3000, 8193), (5, 100, 40000), (1, 0, 10)])
@pytest.mark.parametrize("prompt", [False, True])
def test_counts(hb, B, n, V, prompt):
    rng = np.random.default_rng(n + V)
    tokens = rng.integers(0, V, (B, n)).astype(np.int32)
    length = rng.integers(0, n + 1, B).astype(np.int32)
    start = (rng.integers(0, 4, (B, V)) * (rng.random((B, V)) < 0.3)).astype(np.int32)
    for kw in (dict(), dict(reset=True), dict(length=length), dict(length=length, reset=True),
               dict(index=rng.integers(0, max(n, 1), (B, 7)).astype(np.int32), length=rng.integers(0, 8 if n else 1, B).astype(np.int32))):
        counts = torch.from_numpy(start).cuda()
        dev = {k: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for k, v in kw.items()}
        st = hb.count_tokens(torch.from_numpy(tokens).cuda(), counts, prompt=prompt, **dev)
        want, status = qo.count_tokens(tokens, start, prompt=prompt, **kw)
        assert st.tolist() == status.tolist() == [0] * B
        assert np.array_equal(host(counts), want), kw


def test_counts_out_of_range_are_reported(hb):
    V = 9000
    tokens = torch.tensor([[1, 2, 3], [1, V, 8999], [1, 2, -1], [4, 5, 6], [4, 5, 6]], dtype=torch.int32, device="cuda")
    length = torch.tensor([3, 3, 3, 4, -1], dtype=torch.int32, device="cuda")
    start = torch.randint(0, 5, (5, V), dtype=torch.int32, device="cuda")
    for reset in (False, True):
        counts = start.clone()
        st = hb.count_tokens(tokens, counts, length=length, reset=reset)
        want, status = qo.count_tokens(host(tokens), host(start), length=host(length), reset=reset)
        assert st.tolist() == status.tolist() == [0, 7, 7, 7, 7] and np.array_equal(host(counts), want)
    index = torch.tensor([[0, 3], [2, -1], [0, 1], [1, 1], [0, 0]], dtype=torch.int32, device="cuda")
    counts = start.clone()
    st = hb.count_tokens(tokens, counts, index=index)
    want, status = qo.count_tokens(host(tokens), host(start), index=host(index))
    assert st.tolist() == status.tolist() == [7, 7, 0, 0, 0] and np.array_equal(host(counts), want)


@pytest.mark.parametrize("in_place", [False, True], ids=["apart", "in_place"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_a_block(hb, dtype, in_place):
    """Batches large enough for a warp to take several rows, one after the other: the next row's mask and logits are on their way
    while one is worked on, in the same places."""
    c = Case(9, dtype, 16, 128, 2, 20001, seen=900, n_bias=40, masked=True)
    c.check(hb, in_place)
    c.check(hb, in_place, allowed=None)
