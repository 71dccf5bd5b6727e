"""What the 8-bit attention may be given at its edges, and what a call of it promises."""
import numpy as np
import pytest
import torch

from test_gpu_q8_attention import Case, close, hb  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,kw", [((4, 91, 32, 32, 128, (4000, 3800, 4096, 3500)), dict()), ((3, 40, 40, 40, 128, (900, 1000, 1100)), dict()),
                                      ((6, 50, 40, 8, 128, (512, 8000, 700, 3000, 2000, 5000)), dict(window=1024, sinks=4))], ids=["two_parts", "cut", "window"])
def test_a_call_repeats_itself(hb, shape, kw):  # noqa: F811
    """Which CTA delivers the last part of a unit is a matter of timing; the result is not."""
    c = Case(2, "bf16", *shape)
    first = c.run(hb, **kw)[0].view(torch.int16)
    lens, par, more = torch.from_numpy(c.lens).cuda(), torch.from_numpy(c.parent).cuda(), dict(kw, out=torch.empty_like(c.q))
    other = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(1000):
        out, _ = hb.tree_attention_q8(c.q, c.k, c.v, c.ks, c.vs, lens, par, **more)
        other += (out.view(torch.int16) != first).sum()
    assert int(other) == 0


def spare_page(c, unseen):
    """Page 0 becomes the pool's spare page, full of codes that are no numbers under the largest scale; the entries of pages that
    `unseen` (sequence, logical page) names point at it, by their number or by one outside the pool."""
    n = c.k.shape[0]
    free = sorted(set(range(1, n)) - set(c.table.reshape(-1).tolist()))
    c.table[c.table == 0] = free[0]
    c.upload()
    for t, what in ((c.k, 0x7F), (c.v, 0xFF), (c.ks, 254), (c.vs, 254)):
        t.view(torch.uint8)[0] = what
    for i, (b, page) in enumerate(unseen):
        c.table[b, page] = (0, -1, 1 << 30)[i % 3]


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 128), ("f32", 64), ("f32", 128), ("bf16", 64)])
@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("window,sinks", [(100, 5), (33, 0), (257, 130)])
def test_pages_that_no_row_sees_may_hold_anything(hb, dtype, D, page, window, sinks):  # noqa: F811
    c = Case(40 + page, dtype, 3, 10, 4, 2, D, (500, 700, 61), page=page)
    want = c.want(window=window, sinks=sinks)
    unseen = [(b, i) for b, L in enumerate(c.lens) for i in range(c.table.shape[1])
              if i * page >= sinks and (i + 1) * page <= L - window + 1 or i * page >= L + 10]
    assert len(unseen) >= 10
    spare_page(c, unseen)
    out, st = c.run(hb, window=window, sinks=sinks)
    assert st.tolist() == [0] * 3
    close(out, want)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 128), ("f32", 64)])
def test_rows_that_no_row_sees_may_hold_anything(hb, dtype, D):  # noqa: F811
    """The rows between the first tokens and the farthest that any window reaches, of pages and of tiles that others see."""
    for page in (0, 16, 256):
        for window, sinks in ((100, 5), (300, 0), (20, 140)):
            c = Case(50 + page, dtype, 2, 20, 4, 2, D, (600, 333), page=page)
            want = c.want(window=window, sinks=sinks)
            for b, L in enumerate(c.lens):
                for x, s in zip(c.codes, c.bytes):
                    x[b, :, sinks:L - window + 1], s[b, :, sinks:L - window + 1] = 0x7F, 254
            c.upload()
            out, st = c.run(hb, window=window, sinks=sinks)
            assert st.tolist() == [0, 0]
            close(out, want, (page, window, sinks))


@pytest.mark.parametrize("dtype,D", [("f32", 64), ("f32", 128), ("bf16", 64)])
@pytest.mark.parametrize("roots,N,L,window,sinks", [(60, 200, 0, 4, 4), (40, 300, 0, 5, 9), (33, 100, 1, 1, 4), (130, 300, 20, 30, 50)])
def test_first_tokens_within_a_tree(hb, dtype, D, roots, N, L, window, sinks):  # noqa: F811
    """A row of the tree stands where its depth puts it: behind wide siblings, rows far down the cache are among the first tokens."""
    parent = np.full((1, N), -1, np.int32)
    parent[0, roots:] = np.arange(roots - 1, N - 1)                                     # a chain below the last root
    for page in (0, 16):
        for kw in (dict(), dict(num_splits=3)):
            Case(N, dtype, 1, N, 2, 2, D, (L,), page=page, parent=parent).check(hb, "%s %s" % (page, kw), window=window, sinks=sinks, **kw)
    if dtype == "bf16":                                                                 # the tensor cores
        Case(N, dtype, 1, N, 2, 2, 128, (L,), parent=parent).check(hb, window=window, sinks=sinks)


def test_split_calls_on_the_alus_leave_a_workspace_clean(hb):  # noqa: F811
    """Calls with parts of their own, of the 8-bit and of the other caches, between calls that count on the counters' area."""
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    clean = [Case(20, "bf16", 3, 40, 40, 40, 128, (900, 1000, 1100)), Case(23, "f16", 6, 5, 16, 16, 128, (700, 1, 300, 900, 40, 6000))]
    split = [Case(80, "f32", 2, 30, 4, 2, 64, (600, 90)), Case(81, "bf16", 1, 9, 8, 2, 64, (900,), page=16), Case(82, "bf16", 2, 20, 6, 2, 128, (500, 300))]
    want = [c.want() for c in clean + split]
    lens = lambda c: (torch.from_numpy(c.lens).cuda(), torch.from_numpy(c.parent).cuda())  # noqa: E731
    k16 = torch.randn((2, 2, 700, 64), device="cuda")
    def others():                                                                       # the call of 16- and 32-bit caches
        _, st = hb.tree_attention(split[0].q, k16, k16, *lens(split[0]), workspace=ws, num_splits=5)
        assert st.tolist() == [0, 0]
    for between in [lambda c=c, w=w, kw=kw: (c, w, kw) for c, w in zip(split, want[2:]) for kw in (dict(), dict(num_splits=6))] + [others, None]:
        if between is others:
            others()
        elif between:
            c, w, kw = between()
            out, st = c.run(hb, workspace=ws, **kw)
            assert (st == 0).all()
            close(out, w)
        assert int(ws[:65536].view(torch.int32).abs().max()) == 0
        for c, w in zip(clean, want):
            out, st = c.run(hb, workspace=ws, flags=hb.HT_ATTN_WORKSPACE_CLEAN)
            assert (st == 0).all()
            close(out, w)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 128), ("f32", 64), ("f16", 64)])
@pytest.mark.parametrize("shape", [(2, 7, 4, 2, (300, 5)), (1, 20, 8, 8, (1500,)), (4, 33, 40, 40, (500, 17, 260, 900))], ids=["few", "clusters", "list"])
def test_queries_that_are_no_numbers(hb, dtype, D, shape):  # noqa: F811
    """A query row with an infinity or a NaN gives NaN, whatever else it holds and whatever it sees; the rows next to it are what they were."""
    B, N, Hq, Hkv, lens = shape
    for kw in (dict(), dict(window=40, sinks=3)):
        c = Case(60, dtype, B, N, Hq, Hkv, D, lens)
        want = c.want(**kw)
        rng = np.random.default_rng(N)
        hit = np.zeros((B, N, Hq), bool)
        for i in range(3 * B):
            b, r, h = rng.integers(B), rng.integers(N), rng.integers(Hq)
            c.q[b, r, h, int(rng.integers(D))] = (float("inf"), -float("inf"), float("nan"))[i % 3]
            hit[b, r, h] = True
        c.q[0, 0, 0], hit[0, 0, 0] = float("inf"), True
        out, st = c.run(hb, **kw)
        assert st.tolist() == [0] * B
        assert np.array_equal(out.isnan().any(-1).cpu().numpy(), hit) and np.array_equal(out.isnan().all(-1).cpu().numpy(), hit)
        close(out, tuple(np.where(hit[..., None], np.nan, w) for w in want), str(kw))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_queries_on_zero_keys(hb, dtype):  # noqa: F811
    """Scores that vanish next to one another leave equal weights, whatever powers of two they are made of."""
    for power in (-60, -110):
        for zeros in (slice(None), slice(130, None), slice(0, 256)):
            c = Case(70, dtype, 2, 9, 4, 2, 128, (300, 40))
            c.q = (c.q.double() * 2.0 ** power).to(c.q.dtype)
            c.codes[0][:, :, zeros], c.bytes[0][:, :, zeros] = 0, 1
            c.upload()
            c.check(hb, "%d %s" % (power, zeros))
            c.check(hb, "%d %s" % (power, zeros), window=20, sinks=3)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_long_texts_of_zero_values(hb, dtype):  # noqa: F811
    """The sum of the weights of tens of thousands of keys whose values are all zero: one key that is not has its share of the whole.

    Every head holds the same: two tiles of zero keys, 2^15 and more rows that score 7.9 above them in powers of two and hold zeros, and one
    last context row that scores 7.9 too and holds ones.  Result: 1 / (number of those rows + what the others add)."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    N, D, H, L, cap = 1, 128, sms, 46000, 46016
    a = 4.0
    k = torch.zeros((1, H, cap, D), dtype=torch.uint8, device="cuda")
    v, ks, vs = torch.zeros_like(k), torch.full((1, H, cap), 127, dtype=torch.uint8, device="cuda"), torch.ones((1, H, cap), dtype=torch.uint8, device="cuda")
    k[:, :, 256:L, 0] = 0x38                                                            # 1.0 in the first feature
    v[:, :, L - 1] = 0x38
    vs[:, :, L - 1] = 127
    q = torch.zeros((1, N, H, D), dtype=torch.bfloat16 if dtype == "bf16" else torch.float16, device="cuda")
    q[..., 0] = a
    scale = 7.9 * np.log(2.0) / a
    ty = lambda t: t.view(torch.float8_e4m3fn if t.dim() == 4 else torch.float8_e8m0fnu)  # noqa: E731
    out, st = hb.tree_attention_q8(q, ty(k), ty(v), ty(ks), ty(vs), torch.tensor([L], dtype=torch.int32, device="cuda"),
                                   torch.full((1, N), -1, dtype=torch.int32, device="cuda"), scale=scale)
    assert st.tolist() == [0]
    rest = (256 + 1) * 2.0 ** -7.9                                                      # the two tiles, and the row itself (a zero key)
    want = 1.0 / (L - 256 + rest)
    got = out.double()
    # the weight rounded to fp16, the result to the type (fp16: a step of 2^-24 at these sizes), 32-bit sums of 46000 terms by 256 at a time
    half = torch.finfo(out.dtype).eps / 2
    tol = want * (2.0 ** -11 + half + 1e-4) + (2.0 ** -25 if dtype == "f16" else 0.0)
    assert (got - want).abs().max() <= tol, (got.min(), got.max(), want)


def test_windows_beyond_32_bits_are_refused(hb):  # noqa: F811
    c = Case(90, "bf16", 1, 4, 2, 2, 128, (40,), page=16)
    d = Case(91, "bf16", 1, 4, 2, 2, 128, (40,))
    for case in (c, d):
        for kw in (dict(window=1 << 32), dict(window=(1 << 32) + 5), dict(window=5, sinks=1 << 32), dict(window=5, sinks=(1 << 33) + 1)):
            with pytest.raises(ValueError):
                case.run(hb, **kw)
        case.check(hb, window=(1 << 31) - 1, sinks=(1 << 31) - 1)


@pytest.mark.parametrize("shape,page", [((2, 40, 40, 40, 128, (2000, 1500)), 0), ((2, 40, 40, 40, 128, (2000, 1500)), 16), ((1, 91, 8, 8, 128, (6000,)), 0),
                                        ((1, 91, 8, 8, 128, (6000,)), 64), ((3, 67, 64, 8, 128, (3000, 2000, 900)), 128)],
                         ids=["list", "list_paged", "clusters", "clusters_paged", "groups_paged"])
def test_waits_that_run_out_are_reported_in_every_form(hb, shape, page):  # noqa: F811
    """The hook that lets no wait last: the calls return, every sequence's status says so, and the next call on the same workspace and
    output is right."""
    c = Case(33, "bf16", *shape, page=page)
    want = c.want()
    ws, out = torch.zeros(48 << 20, dtype=torch.uint8, device="cuda"), torch.empty_like(c.q)
    for _ in range(3):
        _, st = c.run(hb, flags=hb.HT_ATTN_TEST_SHORT_WAITS, workspace=ws, out=out)
        assert st.tolist() == [hb.HT_STATUS_TIMEOUT] * shape[0]
    for kw in (dict(), dict(flags=hb.HT_ATTN_WORKSPACE_CLEAN)):
        _, st = c.run(hb, workspace=ws, out=out, **kw)
        assert st.tolist() == [0] * shape[0]
        close(out, want, str(kw))
