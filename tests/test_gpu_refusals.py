"""Refusals of the binding that are reached with tensors on a device."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_every_entry_refuses_unsupported_types():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2404_12022_b200 import binding as hb
    z = lambda *s, t=torch.float64: torch.zeros(s, dtype=t, device="cuda")              # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")                     # noqa: E731
    u = torch.zeros((1, 4), device="cuda")
    q, c, pool, table = z(1, 4, 2, 128), z(1, 2, 32, 128), z(2, 2, 16, 128), i(1, 2)
    head = hb.make_head_desc(128)
    for call in (lambda: hb.norm_rope_kv_append(q, q, q, i(1, 4), i(1), c, c, head),
                 lambda: hb.norm_rope_kv_append_paged(q, q, q, i(1, 4), i(1), table, pool, pool, head),
                 lambda: hb.tree_attention_scored(q, c, c, i(1), i(1, 4), cap=1.0),
                 lambda: hb.tree_attention_scored_paged(q, pool, pool, table, i(1), i(1, 4), cap=1.0),
                 lambda: hb.tree_attention(q, c, c, i(1), i(1, 4)),
                 lambda: hb.tree_attention_paged(q, pool, pool, table, i(1), i(1, 4)),
                 lambda: hb.sample(z(1, 4, 50), u),
                 lambda: hb.verify_sampled(z(1, 4, 50), u, i(1, 4), i(1, 4)),
                 lambda: hb.verify_greedy(z(1, 4, 50), i(1, 4), i(1, 4), None, 8)):
        with pytest.raises(ValueError, match="not supported"):
            call()


def test_calls_without_rows_report_nothing():
    """No rows, no status words written: the ones returned must not be what the memory held."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2404_12022_b200 import binding as hb
    B, H, D = 3, 2, 128
    z = lambda *s, t=torch.float16: torch.zeros(s, dtype=t, device="cuda")              # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")                     # noqa: E731
    q, c, pool, table, lens = z(B, 0, H, D), z(B, H, 32, D), z(6, H, 16, D), i(B, 2), i(B)
    rows, u = i(B, 0), torch.zeros((B, 0), device="cuda")
    head = hb.make_head_desc(D)
    for call in (lambda: hb.norm_rope_kv_append(q, q, q, rows, lens, c, c, head),
                 lambda: hb.norm_rope_kv_append_paged(q, q, q, rows, lens, table, pool, pool, head),
                 lambda: hb.tree_attention_scored(q, c, c, lens, rows, cap=1.0),
                 lambda: hb.tree_attention_scored_paged(q, pool, pool, table, lens, rows, cap=1.0),
                 lambda: hb.sample(z(B, 0, 50), u)):
        held = [torch.full((B,), 7, dtype=torch.int32, device="cuda") for _ in range(64)]     # what the allocator hands out next
        torch.cuda.synchronize()
        del held
        out, status = call()
        assert out.shape[:2] == (B, 0) and status.tolist() == [0] * B
    # without sequences there is nothing at all
    assert hb.sample(z(0, 4, 50), torch.zeros((0, 4), device="cuda"))[1].numel() == 0
    assert hb.tree_attention_scored(z(0, 4, H, D), z(0, H, 32, D), z(0, H, 32, D), i(0), i(0, 4), cap=1.0)[0].numel() == 0
