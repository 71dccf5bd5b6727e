"""What the first calls of a program set up on the device."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

CHILD = """
import sys
sys.path.insert(0, %r)
import torch
from paper_2404_12022_b200 import binding as hb
for Hq, N in ((4, 18), (16, 67)):                        # one tile of query rows per KV head, and several
    q = torch.zeros((1, N, Hq, 128), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((1, 2, 200, 128), dtype=torch.bfloat16, device="cuda")
    lens = torch.tensor([100], dtype=torch.int32, device="cuda")
    parent = torch.arange(-1, N - 1, dtype=torch.int32, device="cuda")[None].contiguous()
    pos = torch.arange(100, 100 + N, dtype=torch.int32, device="cuda")[None].contiguous()
    hb.tree_attention(q, k, k, lens, parent)
    print("PLAIN DONE", file=sys.stderr, flush=True)
    hb.tree_attention_scored(q, k, k, lens, parent, cap=30.0)
    hb.tree_attention_scored(q, k, k, lens, parent, slopes=torch.ones(Hq, device="cuda"), pos=pos)
    hb.tree_attention_scored(q, k, k, lens, parent, cap=30.0)
torch.cuda.synchronize()
"""


def test_a_call_sets_up_the_kernels_of_its_own_shape_alone():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CHILD % root], capture_output=True, text=True, timeout=300, env=dict(os.environ, HT_LOG="1"))
    assert r.returncode == 0, r.stderr[-2000:]
    seen = [line.split("kernels set up: scores ")[1].strip() if "set up" in line else "|" for line in r.stderr.splitlines()
            if "kernels set up" in line or "PLAIN DONE" in line]
    assert seen == ["plain", "|", "capped", "biased"] * 2, r.stderr[-2000:]


CAPTURE = """
import sys
sys.path.insert(0, %r)
import torch
from paper_2404_12022_b200 import binding as hb
torch.cuda.init()
for Hq, N in ((4, 18), (16, 67)):
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()
    q, k, v = rnd(1, N, Hq, 128), rnd(1, 2, 200, 128), rnd(1, 2, 200, 128)
    lens = torch.tensor([100], dtype=torch.int32, device="cuda")
    parent = torch.arange(-1, N - 1, dtype=torch.int32, device="cuda")[None].contiguous()
    pos = torch.arange(100, 100 + N, dtype=torch.int32, device="cuda")[None].contiguous()
    slopes = torch.full((Hq,), 0.1, device="cuda")
    ws = torch.zeros(48 << 20, dtype=torch.uint8, device="cuda")
    x, u = rnd(1, N, 9000), torch.rand((1, N), generator=g, device="cuda")
    kc, vc = torch.zeros_like(k), torch.zeros_like(v)
    kn, head = rnd(1, N, 2, 128), hb.make_head_desc(128)
    calls = [lambda kw=kw: hb.tree_attention_scored(q, k, v, lens, parent, workspace=ws, **kw)[0]
             for kw in (dict(cap=30.0), dict(slopes=slopes, pos=pos), dict(cap=30.0, slopes=slopes, pos=pos), dict())]
    calls += [lambda: hb.sample(x, u)[0], lambda: hb.norm_rope_kv_append(q, kn, kn, pos, lens, kc, vc, head)[0]]
    for call in calls:
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            out = call()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call())
print("ALL CAPTURED")
"""


def test_a_process_may_capture_its_first_call_of_a_kind():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CAPTURE % root], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "ALL CAPTURED" in r.stdout, r.stderr[-2000:]
