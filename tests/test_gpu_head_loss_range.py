"""Logits far from zero, of single products that float32 holds exactly: up to 1.8e8 (bf16 operands) and 7e8 (float32)
the losses and gradients are the formulas', beyond that the row is NaN and flagged; a part of the vocabulary far below
the rest is nothing but p = 0."""
import pytest
import torch

import paper_2607_07508_amd as sao
from paper_2607_07508_amd import binding
from tests.gpu_common import say
from tests.head_loss_exact import DT, check_grad, head_loss

pytestmark = pytest.mark.gpu

H = 64
SIZES = [(48, 5000), (300, 50257), (700, 33001)]   # few rows; one token tile; three


def single_products(T, V, dtype, seed, factors):
    """z = h[t, 0] w[v, 0]: 7 and 2 significand bits, so exact; the largest of a row differs from the next by 2^-8 of it
    or more, or equals it. The other columns of h meet zeros of w and show in dw."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn((T, H), generator=g, device="cuda")
    w = torch.zeros((V, H), device="cuda")
    w[:, 0] = 2048 + 16 * torch.randint(0, 100, (V,), generator=g, device="cuda").float()
    h[:, 0] = torch.tensor(factors, device="cuda")[torch.randint(0, len(factors), (T,), generator=g, device="cuda")]
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    y[::2] = (h[:, :1].double() @ w[:, :1].double().t()).argmax(1).to(torch.int32)[::2]
    return h.to(DT[dtype]), w.to(DT[dtype]), y


def check(out, ref, dtype):
    loss, token, lse, dh, dw = out
    # the scale log2 e is a float and lse one too: both 2^-24 of the largest logit, and 2^-23 of theirs
    bar = 2.0 ** -22 * ref["z"] + 2e-5
    assert float((lse.double() - ref["lse"]).abs().max()) <= bar
    assert float((token.double() - ref["token"]).abs().max()) <= bar
    exact = dict(ref, z=0.0)   # the logits are exact
    check_grad(dh, exact, "dhidden", H, dtype)
    check_grad(dw, exact, "dw", H, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", SIZES)
def test_large_logits(T, V, dtype):
    say(f"large logits {T} {V} {dtype}")
    # logits up to 1.3e7, 2.6e7, 4e7, 8e7 and 1.6e8, either sign
    sizes = [4096.0, 6144.0, 8192.0, 12288.0, 24576.0, 40960.0]
    h, w, y = single_products(T, V, dtype, T, sizes + [-s for s in sizes])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = sao.cross_entropy(h, w, y, status=status)
    assert int(status) == 0
    check(out, head_loss(h, w, torch.full((T,), 1.0 / T, device="cuda"), target=y), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", SIZES)
@pytest.mark.parametrize("tau", [2.0 ** -17, 1e-5])
def test_small_temperature(T, V, dtype, tau):
    """Ordinary logits at a temperature of some 1e-5: z / tau is up to 1.4e8, by 1e-5 with a rounding of its own."""
    say(f"small temperature {T} {V} {dtype} {tau}")
    h, w, y = single_products(T, V, dtype, T + 1, [0.0625, 0.125, 0.1875, 0.25, -0.0625, -0.25])
    ids = torch.stack([y, (y + 11) % V, (y + 500) % V], 1).to(torch.int32).contiguous()
    teacher = torch.tensor([3.0, 2.0, 1.0], device="cuda").expand(T, 3).contiguous() * tau
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, token, lse, dh, dw = sao.distill_loss(h, w, ids, teacher, temperature=tau, status=status)
    assert int(status) == 0
    ref = head_loss(h, w, torch.full((T,), 1.0 / T, device="cuda"), ids=ids, teacher=teacher, tau=tau)
    assert float((lse.double() - ref["lse"]).abs().max()) <= 2.0 ** -22 * ref["z"]
    assert float((token.double() - ref["token"]).abs().max()) <= tau ** 2 * (2.0 ** -22 * ref["z"] + 2e-5)
    exact = dict(ref, z=0.0)
    check_grad(dh, exact, "dhidden", H, dtype)
    check_grad(dw, exact, "dw", H, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", SIZES)
def test_a_part_far_below(T, V, dtype):
    """512 vocabulary rows hundreds of millions below ordinary ones, each half tile of them at a distance of its own."""
    say(f"part far below {T} {V} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(T + 2)
    h = torch.randn((T, H), generator=g, device="cuda")
    w = torch.randn((V, H), generator=g, device="cuda") * 0.25
    w[:, 0] = 0.0
    w[256:768, 0] = -(2048 + 16 * torch.arange(512, device="cuda") // 8).float()
    w[256:768, 1:] = 0.0
    # the last: products of up to -2.5e38, which log2 e takes out of float32
    h[:, 0] = torch.tensor([2.0 ** k for k in (*range(10, 21), 116)], device="cuda")[torch.arange(T, device="cuda") % 12]
    h, w = h.to(DT[dtype]), w.to(DT[dtype])
    y = torch.randint(1000, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = sao.cross_entropy(h, w, y, status=status)
    assert int(status) == 0
    ref = head_loss(h, w, torch.full((T,), 1.0 / T, device="cuda"), target=y)
    ref["z"] = 40.0   # of the rows that have a probability
    check_grad(out[3], ref, "dhidden", H, dtype)
    check_grad(out[4], ref, "dw", H, dtype)
    assert float((out[1].double() - ref["token"]).abs().max()) <= 1e-4


@pytest.mark.parametrize("dtype,size", [("bf16", 2.0 ** 17), ("bf16", 2.0 ** 40), ("f32", 2.0 ** 19), ("f32", 2.0 ** 40)])
@pytest.mark.parametrize("T,V", SIZES)
def test_beyond_the_range_is_flagged(T, V, dtype, size):
    say(f"out of range {T} {V} {dtype} {size}")
    for sign in (1.0, -1.0):
        h, w, y = single_products(T, V, dtype, T + 3, [1.0])
        h[7, 0] = sign * size
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        loss, nll, lse, dh, dw = sao.cross_entropy(h, w, y, status=status)
        assert int(status) & binding.STATUS_NONFINITE
        assert torch.isnan(lse[7]) and torch.isnan(nll[7]) and torch.isnan(loss[0]) and torch.isnan(dh[7]).all()
        rest = torch.arange(T, device="cuda") != 7
        assert torch.isfinite(dh[rest]).all() and torch.isfinite(nll[rest]).all() and torch.isfinite(lse[rest]).all()
