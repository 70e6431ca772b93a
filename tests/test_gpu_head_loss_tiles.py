"""Cross entropy and distillation through the kernels that take calls of hundreds and thousands of rows, at widths of 8 to
64 slabs of K and vocabularies of 130 to 200 tiles, and every gradient element of the shapes where kernels change:
each element is held to its own bar (tests/head_loss_exact.py), so that a wrong row of a rare vocabulary entry or of a
token of small weight shows, which a norm over the whole gradient hides."""
import pytest
import torch

import paper_2607_07508_amd as sao
from paper_2607_07508_amd import binding
from tests.gpu_common import say
from tests.head_loss_exact import DT, check_grad, head_loss, logit_eps
from tests.test_gpu_train_losses import EDGES, SHAPES, make, teacher

pytestmark = pytest.mark.gpu

# One, two, three and five token tiles (K wrapped up to two); loss rows 4 and 16 per block; dW by half and whole tiles
TILES = [(200, 512, 33001), (300, 1024, 50257), (500, 512, 33001), (400, 2048, 33001), (700, 1024, 33001), (1100, 512, 33001)]


def factors(T, m, wt):
    on = torch.ones(T, device="cuda") if m is None else m.float()
    n = on.sum().clamp(min=1)
    return (on if wt is None else on * wt).double() / n


def check(out, ref, c, H, dtype, m, tau=1.0):
    loss, token, lse, dh, dw = out
    eps = logit_eps(H, ref["z"], dtype) + 2.0 ** -21 * ref["z"] + 2e-5
    assert float((lse.double() - ref["lse"]).abs().max()) <= eps
    off = (token.double() - ref["token"]).abs()
    assert float(off.max()) <= 2 * tau ** 2 * eps
    assert abs(float(loss[0]) - float((c * ref["token"]).sum())) <= 2 * tau ** 2 * eps * float(c.abs().sum())
    check_grad(dh, ref, "dhidden", H, dtype)
    check_grad(dw, ref, "dw", H, dtype, {torch.float32: 24, torch.bfloat16: 8}[dw.dtype])
    if m is not None:
        gone = m == 0
        assert not dh[gone].any() and not token[gone].any() and not lse[gone].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,V", TILES + EDGES + SHAPES)
def test_every_element_of_cross_entropy(T, H, V, dtype):
    say(f"elements of cross entropy {T} {H} {V} {dtype}")
    h, w, y, m, wt = make(T, H, V, dtype, T + V, "some", True, pad=8)
    if not bool(m.any()):
        m[-1] = 1
    y[-1] = V - 1                                     # the last row of a partial tile
    wt[: T // 2] *= 1e-3                              # tokens that a norm over all of them would not show
    c = factors(T, m, wt)
    ref = head_loss(h, w, c, target=y, z_coef=1e-3)
    out = sao.cross_entropy(h, w, y, m, weight=wt, z_coef=1e-3)
    check(out, ref, c, H, dtype, m)
    # added to a float32 accumulator: the same sums, not rounded to the operands' type
    acc = torch.zeros((V, H), device="cuda")
    loss = torch.zeros(2, dtype=torch.float64, device="cuda")
    check(sao.cross_entropy(h, w, y, m, weight=wt, z_coef=1e-3, loss=loss, dw_head=acc), ref, c, H, dtype, m)
    only = sao.cross_entropy(h, w, y, m, weight=wt, z_coef=1e-3, want_dhidden=False, want_dw=False)
    assert all(torch.equal(a, b) for a, b in zip(only[:3], out[:3])) and only[3] is None and only[4] is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,V,K", [(*s, k) for s, k in zip(TILES, (20, 64, 5, 256, 1, 33))] +
                         [(40, 264, 5000, 20), (65, 72, 16500, 5), (4097, 72, 400, 7)])
def test_every_element_of_distillation(T, H, V, K, dtype):
    say(f"elements of distillation {T} {H} {V} {K} {dtype}")
    h, w, _, m, wt = make(T, H, V, dtype, T + V + 1, "some", True, pad=8)
    ids, t, _ = teacher(T, V, K, T + K, False)
    wt[: T // 2] *= 1e-3
    c = factors(T, m, wt)
    for tau in (1.0, 2.0):
        ref = head_loss(h, w, c, ids=ids, teacher=t, tau=tau)
        out = sao.distill_loss(h, w, ids, t, m, weight=wt, temperature=tau)
        check(out, ref, c, H, dtype, m, tau)
        only = sao.distill_loss(h, w, ids, t, m, weight=wt, temperature=tau, want_dhidden=False, want_dw=False)
        assert all(torch.equal(a, b) for a, b in zip(only[:3], out[:3])) and only[3] is None and only[4] is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,V", [(3, 64, 1000), (40, 72, 5000), (300, 128, 20000), (1100, 128, 9000), (17409, 64, 151936)])
def test_stored_float32_weight_gradient(T, H, V, dtype):
    """The C entry points' form that overwrites the loss and a float32 dw_head, over what the arrays held before, in one
    chunk of rows and in two: what adding to zeros gives, to the last bit; and zeros when no token counts."""
    say(f"stored dw {T} {H} {V} {dtype}")
    h, w, y, m, _ = make(T, H, V, dtype, T + H, "some", False)
    ids, t, _ = teacher(T, V, 3, T, False) if T < 5000 else (None, None, None)
    L, dt = binding.lib(), {"bf16": binding.SAO_BF16, "f32": binding.SAO_F32}[dtype]
    stream = torch.cuda.current_stream().cuda_stream

    def stored(K, mask):
        ws = torch.empty(L.sao_head_loss_workspace_size(T, H, V, max(K, 1), dt, binding.OUT_STORE, 1, 1), dtype=torch.uint8,
                         device="cuda")
        loss = torch.full((2,), 7.0, dtype=torch.float64, device="cuda")
        token, lse = torch.full((2, T), 7.0, device="cuda")
        dh = torch.full((T, H), 7.0, dtype=DT[dtype], device="cuda")
        dw = torch.full((V, H), float("nan"), device="cuda")
        if K:
            s = L.sao_distill_loss(h.data_ptr(), H, w.data_ptr(), H, ids.data_ptr(), ids.stride(0), t.data_ptr(), t.stride(0),
                                   None, mask.data_ptr(), None, T, H, V, K, dt, 1.0, None, binding.OUT_STORE, loss.data_ptr(),
                                   token.data_ptr(), lse.data_ptr(), dh.data_ptr(), dw.data_ptr(), None, ws.data_ptr(),
                                   ws.numel(), stream)
        else:
            s = L.sao_cross_entropy(h.data_ptr(), H, w.data_ptr(), H, y.data_ptr(), mask.data_ptr(), None, T, H, V, dt, 1e-3,
                                    None, binding.OUT_STORE, loss.data_ptr(), token.data_ptr(), lse.data_ptr(), dh.data_ptr(),
                                    dw.data_ptr(), None, ws.data_ptr(), ws.numel(), stream)
        assert s == 0
        return loss, token, lse, dh, dw

    acc, loss = torch.zeros((V, H), device="cuda"), torch.zeros(2, dtype=torch.float64, device="cuda")
    added = sao.cross_entropy(h, w, y, m, z_coef=1e-3, loss=loss, dw_head=acc)
    assert all(torch.equal(a, b) for a, b in zip(stored(0, m), added))
    none = torch.zeros_like(m)
    assert not any(x.any() for x in stored(0, none))
    if ids is None:
        return
    acc, loss = torch.zeros((V, H), device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda")
    added = sao.distill_loss(h, w, ids, t, m, loss=loss, dw_head=acc)
    got = stored(3, m)
    assert torch.equal(got[0][:1], added[0]) and float(got[0][1]) == 7.0
    assert all(torch.equal(a, b) for a, b in zip(got[1:], added[1:]))
