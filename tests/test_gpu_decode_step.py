"""The operators of a decode step together, as the example runs them.  Against float32 with unquantized weights the branch is off by what
4-bit weights cost (relative error of a normal block 0.1 to 0.12 per product: two in a row, and once more through keys and values) and
the cache's format (E2M1 the same again, E4M3 0.02 to 0.04)."""
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
