"""The expert block: grouped, gathered and combined, against each expert's dense layer on its own rows."""
import pytest
import torch

from paper_2608_01653_gb300 import hatq as H
from paper_2608_01653_gb300.experts import ExpertBlock, plan

pytestmark = pytest.mark.gpu


def block(experts, c, f, hb_in, hb_mid, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    up = (torch.randn(experts, 2 * f, c, generator=g, device="cuda") * c ** -0.5).to(dtype)
    down = (torch.randn(experts, c, f, generator=g, device="cuda") * f ** -0.5).to(dtype)
    return up, down, ExpertBlock(up, down, hb_in, hb_mid)


@pytest.mark.parametrize("tokens,topk", [(1, 2), (3, 4), (40, 2), (300, 3)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_block_equals_its_experts(tokens, topk, dtype):
    experts, c, f, hb_in, hb_mid = 6, 256, 192, 128, 64
    up, down, B = block(experts, c, f, hb_in, hb_mid, dtype, 1)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(tokens, c, generator=g, device="cuda").to(dtype)
    ids = torch.randint(0, experts + 1, (tokens, topk), generator=g, device="cuda")    # the last one is no expert
    weights = torch.rand(tokens, topk, generator=g, device="cuda")
    y = B.forward(x, ids, weights)
    torch.cuda.synchronize()
    H.sync_status()
    assert y.dtype == dtype and y.shape == (tokens, c)
    # every expert's dense layer on all tokens; the sums are exact, so rows do not depend on what they are grouped with
    ref, size = torch.zeros(tokens, c, dtype=torch.float64, device="cuda"), torch.zeros(tokens, c, dtype=torch.float64, device="cuda")
    for e in range(experts):
        q, s = H.quantize_tokens(x, hb=hb_in)
        h = H.linear(q, s, H.prepare_linear(up[e], hb=hb_in), dtype=dtype)
        q, s = H.quantize_tokens(h, hb=hb_mid, act="silu", gated=True)
        z = H.linear(q, s, H.prepare_linear(down[e], hb=hb_mid), dtype=dtype).double()
        w = torch.where(ids == e, weights, 0.0).double().sum(1, keepdim=True)
        ref += w * z
        size += w * z.abs()
    # topk + 1 fp32 roundings of the sum, one to the output type
    tol = (topk + 1) * 1.01 * 2.0 ** -24 * size + 1.01 * (torch.finfo(dtype).eps / 2 if dtype != torch.float32 else 0) * ref.abs()
    assert bool(((y.double() - ref).abs() <= tol + 2.0 ** -60).all())


def test_block_follows_the_float_layer_and_captures():
    experts, c, f, topk, tokens = 4, 512, 256, 2, 64
    up, down, B = block(experts, c, f, 128, 128, torch.float32, 3)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(tokens, c, generator=g, device="cuda")
    ids = torch.stack([torch.randperm(experts, generator=g, device="cuda")[:topk] for _ in range(tokens)])
    weights = torch.softmax(torch.randn(tokens, topk, generator=g, device="cuda"), 1)

    def float_layer(v):
        h = torch.einsum("tc,ekc->tek", v.double(), up.double())
        u = torch.nn.functional.silu(h[..., :f]) * h[..., f:]
        z = torch.einsum("tef,ecf->tec", u, down.double())
        return (torch.gather(z, 1, ids[:, :, None].expand(-1, -1, c)) * weights.double()[:, :, None]).sum(1)

    y = B.forward(x, ids, weights)
    # four operands in 8 bits with a step of about max / 127: some percent of the result, far below a wrong row's 100 %
    assert float((y - float_layer(x)).norm() / float_layer(x).norm()) < 0.06
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = B.forward(x, ids, weights)
    x.copy_(torch.randn(tokens, c, generator=g, device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    H.sync_status()
    assert torch.equal(out, B.forward(x, ids, weights))


def test_plan_on_the_device_equals_the_host():
    ids = torch.randint(-1, 9, (100, 4), generator=torch.Generator().manual_seed(5))
    for a, b in zip(plan(ids, 8), plan(ids.cuda(), 8)):
        assert torch.equal(a, b.cpu())


def test_bad_shapes():
    w = torch.zeros(2, 8, 4, device="cuda")
    with pytest.raises(ValueError):
        ExpertBlock(w, torch.zeros(2, 4, 5, device="cuda"), 1, 1)
