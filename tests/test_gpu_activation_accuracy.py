"""The activations of the fp32 products and their derivatives by themselves: pre-activations that are exact (products with a one and
zeros), so that what is off is the activation's own error, in half steps of fp32."""
import pytest
import torch

import linear_forms as F
from operator_refs import U32, activation, assert_within
from paper_2406_00023_amd import binding as B

pytestmark = pytest.mark.gpu
ROWS, WIDTH = 4096, 8
# hardware exponential 2 and reciprocal 2 (an ulp each); with the rounding of 1 + e, and the two of the correction for the exponent's own
# rounding, a sigmoid is off by 7.  Phi: what the fit is off 3, its argument 3 (which its value follows with a power of 2 at most), its
# last steps and products 5, the exponential 4
SIGMOID, PHI, EXP = 7, 20, 4


def _points(act):
    most = 12.0 if act == "gelu" else 80.0                     # (beyond, results leave the normal numbers)
    a = torch.empty(ROWS, WIDTH).uniform_(-most, most, generator=torch.Generator().manual_seed(3))
    a[:64] = torch.linspace(-4, 4, 64 * WIDTH).reshape(64, WIDTH)
    a[64] = 0
    return a


@pytest.mark.parametrize("act", ["silu", "gelu", "swiglu"])
def test_forward(act):
    a = _points(act)
    x, w = torch.zeros(ROWS, WIDTH), torch.eye(WIDTH).reshape(1, WIDTH, WIDTH)
    x.copy_(a)
    glu = act == "swiglu"
    cfg = B.make_linear_config(ROWS, WIDTH, WIDTH, 1, torch.float32, act=F.ACT[act])
    y, up = torch.empty(ROWS, WIDTH, device="cuda"), torch.flip(w, [1]).contiguous()
    B.etr_expert_linear(cfg, x.cuda(), None, w.cuda(), y, w_up=up.cuda() if glu else None)
    torch.cuda.synchronize()
    b = torch.flip(a, [1]).double()
    want = activation(act, a.double(), b if glu else None)
    assert_within(y, want, ((PHI if act == "gelu" else SIGMOID) + 1 + glu) * U32 * want.abs() + 1e-36, act)


@pytest.mark.parametrize("act", ["silu", "gelu", "swiglu"])
def test_derivative(act):
    a = _points(act)
    glu = act == "swiglu"
    eye, zero = torch.eye(WIDTH).reshape(1, WIDTH, WIDTH).cuda(), torch.zeros(1, WIDTH, WIDTH).cuda()
    cfg = B.make_linear_config(ROWS, WIDTH, WIDTH, 1, torch.float32, act=F.ACT[act])
    ws = B.alloc_workspace(B.etr_linear_workspace_bytes(cfg))
    d = torch.empty(ROWS, WIDTH).uniform_(0.5, 2.0, generator=torch.Generator().manual_seed(4))
    up = torch.flip(a, [0])
    v, dd = a.double(), d.double()
    sig = 1 / (1 + torch.exp(-v))
    if act == "gelu":
        phi = torch.exp(-0.5 * v * v) * 0.39894228040143267794
        cdf = 0.5 * torch.special.erfc(-v / 2 ** 0.5)
        want = dd * (cdf + v * phi)
        bound = (PHI + 2) * cdf + (EXP + 5) * v.abs() * phi
    else:
        # 1 - sigmoid is off by as much as the sigmoid and half a step of 1; then a product with |a|, a sum, a product
        want = dd * sig * (1 + v * (1 - sig)) * (up.double() if glu else 1)
        bound = sig * (SIGMOID + 4) * (1 + (v * (1 - sig)).abs()) + sig * v.abs() * (SIGMOID * sig + 1)
        bound = bound * (up.double().abs() if glu else 1)
    half = [(eye, zero, want, bound)]
    if glu:
        half.append((zero, eye, dd * v * sig, (SIGMOID + 3) * (v * sig).abs()))
    for w, w_up, want, bound in half:
        dx = torch.empty(ROWS, WIDTH, device="cuda")
        B.etr_expert_linear_backward(cfg, None, None, w, d.cuda(), ws, w_up=w_up if glu else None, pre=a.cuda(), pre_up=up.cuda() if glu else None, dx=dx)
        torch.cuda.synchronize()
        assert_within(dx, want, U32 * dd * bound + 1e-36, act)
