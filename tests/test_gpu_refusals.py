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
