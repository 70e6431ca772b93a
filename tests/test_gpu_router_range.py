"""The router's balance loss with logits of every finite size: rows of nothing but the type's lowest value (experts
masked by it), of its largest, and both in one row; infinite ones next to them."""
import numpy as np
import pytest
import torch

import paper_2607_07508_amd as sao
from oracle import train_losses as tl
from tests.gpu_common import say

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,E", [(40, 24), (33, 60), (900, 128), (1500, 250)])
def test_rows_of_extreme_values(T, E, dtype, score):
    """Tokens hold equal extreme logits, so p is 1 / n over them: each gradient element and the loss within the
    arithmetic's 1e-5, and one rounding of the output. One block does the small sizes, four launches the large ones."""
    say(f"router extremes {T} {E} {dtype} {score}")
    k = 3
    g = torch.Generator(device="cuda").manual_seed(T + E)
    x = torch.randn((T, E), generator=g, device="cuda").to(DT[dtype])
    low, high = torch.finfo(DT[dtype]).min, torch.finfo(DT[dtype]).max
    x[0] = low                                  # every expert masked by the lowest value
    x[1] = high
    x[2] = low
    x[2, ::3] = high
    x[3, ::2] = low                             # some masked, ordinary ones left
    x[4] = low
    x[4, 5] = float("-inf")                     # not offered, among masked ones
    x[5] = 0.75 * low
    x[6] = 3.0e38
    x[6, 1] = 1.5e38
    ids = torch.stack([torch.randperm(E, generator=g, device="cuda")[:k] for _ in range(T)]).to(torch.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, counts, dx = sao.balance_loss(x, ids, coef=1.0, score=score, status=status)
    assert int(status) == 0
    with np.errstate(over="ignore"):
        ref = tl.balance_loss(x.double().cpu().numpy(), ids.cpu().numpy(), coef=1.0, score=score)
    assert np.array_equal(counts.cpu().numpy(), ref["counts"])
    assert abs(float(loss) - ref["loss"][0]) <= 1e-5 * max(1.0, abs(ref["loss"][0]))
    got, want = dx.double().cpu().numpy(), ref["dlogits"]
    assert np.isfinite(got).all()
    # p (f - sum f p): the difference's terms are at most the largest f
    size = E * ref["counts"].max() / (k * T) / T
    assert (np.abs(got - want) <= 1e-5 * size + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * np.abs(want)).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E", [(60, 64), (4000, 64)])
def test_masked_neighbours_do_not_matter(T, E, score):
    """Tokens that count get the same gradient, to the last bit, whatever the masked tokens beside them hold."""
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((T, E), generator=g, device="cuda")
    ids = torch.topk(x, 4, dim=1).indices.to(torch.int32)
    m = (torch.rand(T, generator=g, device="cuda") < 0.6).to(torch.uint8)
    off = m == 0
    first = [v.clone() for v in sao.balance_loss(x, ids, m, score=score)]
    assert not first[2][off].any()
    for value in (-500.0, 500.0, float("-inf"), float("nan")):
        other = x.clone()
        other[off] = value
        assert all(torch.equal(a, b) for a, b in zip(first, sao.balance_loss(other, ids, m, score=score)))
