"""The operators of a decode step together, as the example runs them.  Against float32 with unquantized weights the branch is off by what
4-bit weights cost (relative error of a normal block 0.1 to 0.12 per product: two in a row, and once more through keys and values) and
the cache's format (E2M1 the same again, E4M3 0.02 to 0.04)."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2607_21446_b200 import binding as kb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", ["16bit", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("axes", [None, (24, 24, 24)])
def test_example_is_near_float32(form, axes):
    from examples.decode_step import run
    r = run(prompt=100, steps=3, form=form, axes=axes)
    assert max(r["errors"]) < 0.5
    assert r["out"].shape == (3, 1152) and bool(torch.isfinite(r["out"].float()).all())
    lengths = r["block"].lengths.tolist()
    assert lengths == [103, 66, 29] and r["keys"].shape == (sum(lengths), 4, 72)
    want = torch.cat([h[1] for h in r["history"]])
    assert float((r["values"].float() - want).norm() / want.norm()) < 0.35


def test_a_step_in_one_graph_equals_its_calls():
    """Captured once, replayed for other tokens: the same bits as the calls one by one."""
    from examples.decode_step import Block, randn
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    block = Block(640, 10, 2, 64, 4, 600, 16, "mxfp4", g)
    x = randn(g, 4, 640)
    prompt = randn(g, 1200, 640)
    offsets = torch.tensor([0, 500, 600, 601, 1200], dtype=torch.int32, device="cuda")
    place = torch.cat([torch.arange(n) for n in (500, 100, 1, 599)]).to(torch.int32).cuda()
    block.prompt(prompt, offsets, place)
    start = block.lengths.clone()
    positions = start[:, None].contiguous()
    want = block.step(x, positions).clone()
    block.lengths.copy_(start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block.step(x, positions)
    keep = x.clone()
    x.zero_()
    graph.replay()
    x.copy_(keep)
    block.lengths.copy_(start)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    assert kb.kroquant_last_device_error() == 0


def test_the_first_calls_of_a_process_may_be_captured():
    """What a call asks of the device once (attributes of kernels, clusters that run at once) is allowed in a capture."""
    code = """
import sys
sys.path.insert(0, sys.argv[1])
import torch
from paper_2607_21446_b200 import binding as kb
from examples.decode_step import Block, randn
g = torch.Generator(device="cuda")
g.manual_seed(5)
K = 4096
x, n, heads = randn(g, 16, K), 640, randn(g, 40, 20, 64)
q = torch.randint(0, 256, (n, K // 2), device="cuda", dtype=torch.uint8, generator=g)
s = torch.full((kb.tiled_scale_bytes(n, K),), 120, device="cuda", dtype=torch.uint8)
f = kb.rotary_frequencies([64])
where = torch.arange(40, device="cuda", dtype=torch.int32)
cache = kb.KVCache.empty(8, 16, 4, 64, "mxfp4")
table = torch.arange(4, device="cuda", dtype=torch.int32)[None]
offsets, start = torch.tensor([0, 40], device="cuda", dtype=torch.int32), torch.zeros(1, device="cuda", dtype=torch.int32)
length = start + 40
def calls():
    y = kb.kroquant_linear_w4a16(x, q, s)
    h = kb.kroquant_rotary(heads, None, where, f)
    kb.kroquant_cache_write(cache, h[:, :4], h[:, 4:8], table, offsets=offsets, starts=start)
    return y, h, kb.kroquant_cache_attention(h[:1], cache, table, length)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = calls()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in got]
assert all(torch.equal(a, b) for a, b in zip(got, calls())), "differs"
assert all(bool(torch.isfinite(t.float()).all()) for t in got)
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code, root], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
