"""The example that runs the block's operators together: its quantized branch stays near the float32 one.  Each of the two products
has both operands in 4 bits with one scale per 32 values (relative error of a normal block 0.1 to 0.12 per operand, so 0.15 per
product), which the gated product carries twice."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_block_example_runs_and_is_near_float32():
    from examples.quantized_block import run
    r = run(tokens=384, width=1152, hidden=1504, experts=4)
    assert r["relative_error"] < 0.4
    assert r["out"].shape == (384, 1152) and bool(torch.isfinite(r["out"].float()).all())
    assert r["moe"].shape == (384, 1152) and bool(torch.isfinite(r["moe"].float()).all())
    assert set(r["grads"]) == {"dx", "dy", "dgate", "dscale", "dshift"}


def test_fused_layer_equals_its_two_calls():
    from examples.quantized_block import dense_layer, randn
    from paper_2607_21446_b200 import binding as kb
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    X, W, bias = randn(g, 300, 1152), randn(g, 640, 1152, gain=0.03), randn(g, 640, dtype=torch.float32)
    layer = dense_layer(W)
    q, s = kb.kroquant_quantize(X, layer.factors, scale_layout="tiled")
    want = kb.kroquant_linear_mxfp4(q, s, layer.w_codes, layer.w_scales, bias=bias, activation="gelu")
    assert torch.equal(layer.fused(X, bias=bias, activation="gelu"), want)
    with pytest.raises(ValueError):
        layer.fused(X[:, :1120].contiguous())
