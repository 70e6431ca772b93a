"""The blockless float64 forms that the GPU tests take their elementwise bars from, against the oracle, and that the bars
notice a single wrong row."""
import numpy as np
import pytest
import torch

from oracle import train_losses as tl
from tests.head_loss_exact import check_grad, head_loss


def data(T=23, H=16, V=70, K=5):
    g = torch.Generator().manual_seed(1)
    h, w = torch.randn((T, H), generator=g), torch.randn((V, H), generator=g)
    y = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    m = (torch.rand(T, generator=g) < 0.7).to(torch.uint8)
    wt = torch.rand(T, generator=g)
    ids = torch.randint(-1, V, (T, K), generator=g, dtype=torch.int32)
    t = torch.randn((T, K), generator=g)
    ids[3], t[4] = -1, -torch.inf
    ids[5, 1] = ids[5, 0]
    return h, w, y, m, wt, ids, t, m.double() * wt / m.sum()


def same(ref, want, token):
    for name, other in (("token", token), ("lse", "lse"), ("dhidden", "dhidden"), ("dw", "dw")):
        assert np.allclose(ref[name].numpy(), want[other], rtol=0, atol=1e-6), name


def test_forms_agree_with_the_oracle():
    h, w, y, m, wt, ids, t, c = data()
    same(head_loss(h, w, c, target=y, z_coef=0.1), tl.cross_entropy(h.numpy(), w.numpy(), y.numpy(), m.numpy(), wt.numpy(), 0.1), "nll")
    for tau in (1.0, 2.5):
        same(head_loss(h, w, c, ids=ids, teacher=t, tau=tau),
             tl.distill_loss(h.numpy(), w.numpy(), ids.numpy(), t.numpy(), m.numpy(), wt.numpy(), tau=tau), "token_loss")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bars_notice_one_row(dtype):
    h, w, y, m, wt, _, _, c = data()
    ref = head_loss(h, w, c, target=y)
    for name, row in (("dhidden", int(m.nonzero()[-1])), ("dw", 69)):
        good = ref[name].to(torch.float32 if dtype == "f32" else torch.bfloat16)
        check_grad(good, ref, name, 16, dtype)
        bad = good.clone()
        bad[row] = 0
        with pytest.raises(AssertionError):
            check_grad(bad, ref, name, 16, dtype)
