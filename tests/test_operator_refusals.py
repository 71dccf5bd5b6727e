"""Host-side refusals of the norm + rotary, scored attention and sampling entry points (nothing is launched, no GPU)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def hb():
    from paper_2404_12022_b200 import binding, build
    build.build()
    binding.load()
    return binding


@pytest.fixture(scope="module")
def ptr():
    buf = (ctypes.c_char * (1 << 16))()
    yield (ctypes.addressof(buf) + 255) // 256 * 256       # aligned host addresses: never dereferenced here
    del buf


def place(hb, p, head, desc=None, q_out=None, **at):
    d = desc or hb.AttnDesc(1, 4, 4, 2, 128, 64, hb.HT_BF16, 0.0, 0, 0, 0, 0)
    a = dict(q_in=p, k_in=p + 8192, v_in=p + 12288, q_weight=p, k_weight=p, pos=p, kv_len=p, q_out=p + 16384 if q_out is None else q_out,
             k_cache=p, v_cache=p, status=p)
    a.update(at)
    return hb.load().ht_norm_rope_kv_append(ctypes.byref(d), None if head is None else ctypes.byref(head), *a.values(), None)


def test_norm_rope_refuses(hb, ptr):
    inv, uns = hb.HT_ERR_INVALID_ARG, hb.HT_ERR_UNSUPPORTED
    ok = lambda **kw: hb.make_head_desc(128, **kw)                                      # noqa: E731
    assert place(hb, ptr, None) == inv
    assert place(hb, ptr, ok(rot_dim=130)) == inv
    assert place(hb, ptr, ok(rot_dim=-2)) == inv
    assert place(hb, ptr, ok(rot_dim=63, interleaved=True)) == inv
    assert place(hb, ptr, ok(rot_dim=24)) == uns                       # half-split: whole 16-byte vectors
    assert place(hb, ptr, ok(norm=4)) == inv
    assert place(hb, ptr, ok(eps=-1.0)) == inv and place(hb, ptr, ok(eps=float("nan"))) == inv
    assert place(hb, ptr, ok(rope_base=1.0)) == inv
    assert place(hb, ptr, ok(scaling=3)) == inv and place(hb, ptr, ok(scaling=-1)) == inv
    assert place(hb, ptr, ok(scaling=hb.HT_ROPE_LINEAR, factor=0.0)) == inv
    assert place(hb, ptr, ok(scaling=hb.HT_ROPE_BY_PARTS, factor=2.0, low=4.0, high=4.0, orig_len=100.0)) == inv
    assert place(hb, ptr, ok(scaling=hb.HT_ROPE_BY_PARTS, factor=2.0, orig_len=0.0)) == inv
    for name in ("q_in", "k_in", "v_in", "pos", "kv_len", "k_cache", "v_cache", "status"):
        assert place(hb, ptr, ok(), **{name: None}) == inv
    for name in ("q_in", "k_in", "v_in", "k_cache", "v_cache", "q_weight", "k_weight"):
        assert place(hb, ptr, ok(), **{name: ptr + 2}) == inv
    for stride in ("q_stride", "k_stride", "v_stride"):
        h = ok()
        setattr(h, stride, 8)
        assert place(hb, ptr, h) == inv                                # smaller than a row
        setattr(h, stride, 4 * 128 + 4)
        assert place(hb, ptr, h) == inv                                # not whole vectors
    assert place(hb, ptr, ok(), q_out=ptr + 16) == inv                 # overlaps q_in without being it
    assert place(hb, ptr, ok(), q_out=ptr + 8192) == inv               # overlaps k_in
    h = ok()
    h.q_stride = 1024
    assert place(hb, ptr, h, q_out=ptr) == inv                         # in place needs a dense q_in
    assert place(hb, ptr, ok(), desc=hb.AttnDesc(1, 65, 4, 2, 128, 64, hb.HT_BF16, 0.0, 0, 0, 0, 0)) == inv
    assert place(hb, ptr, ok(), desc=hb.AttnDesc(0, 4, 4, 2, 128, 64, hb.HT_BF16, 0.0, 0, 0, 0, 0)) == hb.HT_OK


def test_norm_rope_paged_refuses(hb, ptr):
    d = hb.AttnDesc(1, 4, 4, 2, 128, 0, hb.HT_BF16, 0.0, 0, 0, 0, 0)
    head = hb.make_head_desc(128)
    call = lambda pages, table: hb.load().ht_norm_rope_kv_append_paged(                # noqa: E731
        ctypes.byref(d), ctypes.byref(head), ctypes.byref(pages), ptr, ptr + 8192, ptr + 12288, None, None, ptr, ptr, table, ptr + 16384,
        ptr, ptr, ptr, None)
    assert call(hb.PagedDesc(24, 4, 8, 0, 0), ptr) == hb.HT_ERR_INVALID_ARG
    assert call(hb.PagedDesc(16, 4, 8, 0, 0), None) == hb.HT_ERR_INVALID_ARG
    assert call(hb.PagedDesc(16, 0, 8, 0, 0), ptr) == hb.HT_ERR_INVALID_ARG
    assert call(hb.PagedDesc(16, 4, 8, 100, 0), ptr) == hb.HT_ERR_INVALID_ARG


def test_scored_attention_refuses(hb, ptr):
    d = hb.AttnDesc(1, 4, 4, 4, 64, 64, hb.HT_F32, 0.0, 0, 0, 1, 0)
    call = lambda s, desc=d: hb.load().ht_tree_attention_scored(                       # noqa: E731
        ctypes.byref(desc), None if s is None else ctypes.byref(s), None, ptr, ptr, ptr, ptr, ptr, None, 0, ptr, None)
    inv = hb.HT_ERR_INVALID_ARG
    for cap in (-1.0, float("nan"), float("inf")):
        assert call(hb.ScoreDesc(cap, None, None)) == inv
        assert b"cap" in hb.load().ht_last_error_string()
    assert call(hb.ScoreDesc(0.0, ptr, None)) == inv and b"pos" in hb.load().ht_last_error_string()
    assert call(hb.ScoreDesc(30.0, None, None)) == inv and b"NULL" in hb.load().ht_last_error_string()     # q is NULL
    assert call(None) == inv
    empty = hb.AttnDesc(0, 4, 4, 4, 64, 64, hb.HT_F32, 0.0, 0, 0, 1, 0)
    assert call(hb.ScoreDesc(30.0, None, None), empty) == hb.HT_OK
    f32 = hb.AttnDesc(1, 4, 4, 4, 128, 0, hb.HT_F32, 0.0, 0, 0, 0, 0)
    paged = hb.load().ht_tree_attention_scored_paged
    pages = hb.PagedDesc(16, 4, 8, 0, 0)
    s = hb.ScoreDesc(30.0, None, None)
    assert paged(ctypes.byref(f32), ctypes.byref(pages), ctypes.byref(s), *[ptr] * 7, ptr, 0, ptr, None) == hb.HT_ERR_UNSUPPORTED
    s = hb.ScoreDesc(-2.0, None, None)
    assert paged(ctypes.byref(f32), ctypes.byref(pages), ctypes.byref(s), *[ptr] * 7, ptr, 0, ptr, None) == inv


def test_sampling_refuses(hb, ptr):
    lib, inv = hb.load(), hb.HT_ERR_INVALID_ARG
    call = lambda logits=ptr, dtype=hb.HT_F16, B=1, N=1, V=100, u=ptr, token=ptr, status=ptr: lib.ht_sample(   # noqa: E731
        logits, dtype, B, N, V, u, None, None, None, None, token, status, None)
    assert call(logits=None) == inv and call(u=None) == inv and call(token=None) == inv and call(status=None) == inv
    assert call(logits=ptr + 4) == inv and call(dtype=5) == inv and call(V=0) == inv and call(B=-1) == inv and call(N=-1) == inv
    assert call(V=(1 << 30) + 1) == hb.HT_ERR_UNSUPPORTED and call(B=1 << 20, N=1 << 10) == hb.HT_ERR_UNSUPPORTED
    assert call(B=0) == hb.HT_OK and call(N=0) == hb.HT_OK
    ver = lambda T=3, N=4, max_path=8, tokens=ptr, parent=ptr, B=1: lib.ht_verify_sampled(                       # noqa: E731
        ptr, hb.HT_F16, ptr, None, None, None, None, tokens, parent, None, B, N, T, 100, max_path, ptr, ptr, ptr, ptr, ptr, None)
    assert ver(T=0) == inv and ver(T=5) == inv and ver(max_path=0) == inv and ver(max_path=256) == inv
    assert ver(tokens=None) == inv and ver(parent=None) == inv
    assert ver(B=0) == hb.HT_OK


def test_binding_refuses_broadcast_rows_and_caches(hb):
    """A stride of 0 stands for "dense" behind the binding: a broadcast tensor's would be read past its end."""
    import torch
    x = torch.zeros(1, 1, 2, 64)
    rows = lambda t, B, N: hb._rows(t, -1, torch.float32, B, N, 64, "k_in")             # noqa: E731
    assert rows(x, 1, 1) == (2, 128)
    assert rows(torch.zeros(2, 3, 6, 64)[:, :, 1:3], 2, 3) == (2, 6 * 64)
    for B, N in ((2, 3), (1, 3), (2, 1)):
        with pytest.raises(ValueError, match="overlap"):
            rows(x.expand(B, N, 2, 64), B, N)
    with pytest.raises(ValueError, match="overlap"):
        rows(torch.zeros(512).as_strided((1, 3, 2, 64), (512, 64, 64, 1)), 1, 3)
    c = torch.zeros(1, 1, 16, 64)
    pair = lambda t: hb._pair(t, t, -1, torch.float32, "caches")                        # noqa: E731
    assert pair(c)[0] == (1, 1, 16, 64)
    for B, H in ((2, 1), (1, 2), (2, 2)):
        with pytest.raises(ValueError, match="broadcast"):
            pair(c.expand(B, H, 16, 64))


def test_caps_beyond_the_arithmetic_are_refused(hb, ptr):
    """A capped score is squared in 32 bits on its way, and so is a product up to cap / scale: beyond 1.8e19 that gave NaN."""
    inv = hb.HT_ERR_INVALID_ARG
    paged, plain = hb.load().ht_tree_attention_scored_paged, hb.load().ht_tree_attention_scored
    pages = hb.PagedDesc(16, 4, 8, 0, 0)

    def both(cap, scale, D=128):
        d = hb.AttnDesc(1, 4, 4, 4, D, 64, hb.HT_BF16, scale, 0, 0, 0, 0)
        s = hb.ScoreDesc(cap, None, None)
        # (a call that passes the check stops at the NULL q)
        a = plain(ctypes.byref(d), ctypes.byref(s), None, ptr, ptr, ptr, ptr, ptr, None, 0, ptr, None), hb.load().ht_last_error_string()
        b = paged(ctypes.byref(d), ctypes.byref(pages), ctypes.byref(s), None, *[ptr] * 6, ptr, 0, ptr, None), hb.load().ht_last_error_string()
        assert a[0] == b[0] == inv and (b"NULL" in a[1]) == (b"NULL" in b[1])
        return b"NULL" in a[1]
    for cap, scale in ((1.3e19, 0.0), (1e30, 0.0), (1e20, 1e4), (1e17, 1e-2), (1.0, 1e-20), (30.0, 1e5), (30.0, float("inf"))):
        assert not both(cap, scale), (cap, scale)
    for cap, scale in ((8e16, 0.0), (1e18, 1.0), (1e8, 0.0), (50.0, 1e-10), (30.0, 1e4), (1e-6, 0.0)):
        assert both(cap, scale), (cap, scale)
    d = hb.AttnDesc(1, 4, 4, 4, 128, 64, hb.HT_BF16, 1e6, 0, 0, 0, 0)                  # without a cap any scale passes
    s = hb.ScoreDesc(0.0, ptr, ptr)
    assert plain(ctypes.byref(d), ctypes.byref(s), None, ptr, ptr, ptr, ptr, ptr, None, 0, ptr, None) == inv
    assert b"NULL" in hb.load().ht_last_error_string()


def test_unsupported_types_are_refused_like_all_else(hb):
    import torch
    for dtype in (torch.float64, torch.int32, torch.float8_e4m3fn):
        with pytest.raises(ValueError, match="not supported: float32, float16 or bfloat16"):
            hb._DTYPES[dtype]
    assert [hb._DTYPES[t] for t in (torch.float32, torch.float16, torch.bfloat16)] == [hb.HT_F32, hb.HT_F16, hb.HT_BF16]
