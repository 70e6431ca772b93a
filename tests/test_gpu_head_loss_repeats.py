"""Cross entropy and distillation through whole logit tiles repeat to the last bit, whichever workgroup takes a
tile: a call after a call, on another stream, and replayed from a graph; and the target's own logit is the one that the
softmax's sum holds. Up to two token tiles a tile's sum over K starts at a slab of its own, with more at the first."""
import pytest
import torch

import paper_2607_07508_amd as sao
from tests.gpu_common import say

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}

# K of 16 to 64 slabs; one, two and three token tiles; a partial last vocabulary tile
SHAPES = [(200, 1024, 50257), (400, 2048, 33001), (600, 1024, 33001)]


def inputs(T, H, V, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn((T, H), generator=g, device="cuda").to(DT[dtype])
    w = (2 / H ** 0.5 * torch.randn((V, H), generator=g, device="cuda")).to(DT[dtype])
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    m = (torch.rand(T, generator=g, device="cuda") < 0.8).to(torch.uint8)
    ids = (y[:, None] + 97 * torch.arange(6, device="cuda", dtype=torch.int32)) % V
    t = torch.randn((T, 6), generator=g, device="cuda")
    return h, w, y, m, ids.to(torch.int32).contiguous(), t


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,V", SHAPES)
def test_whole_tiles_repeat(T, H, V, dtype):
    say(f"repeats {T} {H} {V} {dtype}")
    h, w, y, m, ids, t = inputs(T, H, V, dtype, T + H)

    def step():
        return [*sao.cross_entropy(h, w, y, m, z_coef=1e-3), *sao.distill_loss(h, w, ids, t, m)]

    first = [x.clone() for x in step()]
    names = ["loss", "nll", "lse", "dhidden", "dw", "distill loss", "kl", "distill lse", "distill dhidden", "distill dw"]

    def same(got, where):
        for a, b, name in zip(first, got, names):
            assert torch.equal(a, b), (where, name, float((a.double() - b.double()).abs().max()))

    for i in range(6):
        same(step(), f"call {i + 2}")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    side.synchronize()
    same(other, "side stream")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        for x in held:
            x.fill_(7)
        torch.randn(1000, device="cuda").sum().item()
        graph.replay()
        torch.cuda.synchronize()
        same(held, f"replay {i + 1}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [40, 200, 400, 600])
def test_a_certain_target_has_no_gradient(T, dtype):
    """Hidden states along their target's row, with every other logit more than 200 below: all other exponentials are 0
    in float32, so p is exactly 1 and the gradient exactly 0 if and only if the target's logit is the summed one."""
    say(f"certain targets {T} {dtype}")
    H, V = 1024, 50257
    g = torch.Generator(device="cuda").manual_seed(T)
    w = (0.02 * torch.randn((V, H), generator=g, device="cuda")).to(DT[dtype])
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    scale = 900 + 300 * torch.rand((T, 1), generator=g, device="cuda")
    h = (scale * w[y.long()].float()).to(DT[dtype])
    z = h.double() @ w.double().t()
    top = z.topk(2, dim=1)
    # a target drawn twice has one row of W, so the runner-up is another vocabulary row
    assert (top.indices[:, 0] == y).all() and float((top.values[:, 0] - top.values[:, 1]).min()) > 200
    _, nll, _, dh, dw = sao.cross_entropy(h, w, y)
    assert torch.isfinite(nll).all()
    assert int((dh != 0).any(1).sum()) == 0, int((dh != 0).any(1).sum())
    assert not dw.any()
