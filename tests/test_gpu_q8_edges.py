"""What the 8-bit attention may be given at its edges, and what a call of it promises."""
import pytest
import torch

from test_gpu_q8_attention import Case, hb  # noqa: F401

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
