"""The residual norm with 8-bit rows against its definition: the rounded results themselves, and rows and weights at the ends of their
range.

The kernel forms n = u / sqrt(mean(u^2) + eps) * weight in 64 bits (sum of at most 8192 squares, root, two products: off by less
than 2^-40 of n) and rounds it to fp32, by 2^-24 at most; the definition allows an evaluation in fp32.  So a result is the
rounding of some number within 2^-23 of n, which is the rounding of n itself unless a border between two roundings lies in
between: for bf16 a share of about 2^-23 / 2^-8 of all values, for 8-bit values 2^-23 / 2^-4."""
import pytest
import torch

from tests import mx_reference as ref
from tests.test_gpu_mx import bits, moe, rows  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

NEAR = 2.0 ** -23


def check_exact(moe, x, y, w, eps, T=None):
    s, out, q, scales = moe.moe_residual_norm_mx(x.cuda(), None if y is None else y.cuda(), None if w is None else w.cuda(), eps)
    u32 = x.float() if y is None else x.float() + y.float()
    u, n = ref.norm(u32, None, w, eps)
    assert torch.equal(bits(s.cpu()), bits(u32.to(torch.bfloat16)))
    lo, hi = n * (1 - NEAR), n * (1 + NEAR)
    a, b = lo.float().to(torch.bfloat16), hi.float().to(torch.bfloat16)      # (n up to the smallest normal bf16: 2^-23 is more than a float's step)
    got = out.cpu()
    assert bool(((got == a) | (got == b)).all())
    assert float((a != b).double().mean()) < 1e-3
    v, e = ref.values((q, scales)), scales.cpu().view(torch.uint8).int() - 127
    (va, ea), (vb, eb) = ref.mx(lo), ref.mx(hi)
    assert bool(((e == ea) | (e == eb)).all())
    sure = (ea == eb).repeat_interleave(32, -1)
    assert bool(((v == va) | (v == vb))[sure].all())
    assert float((~sure | (va != vb)).double().mean()) < 1e-3


@pytest.mark.parametrize("T,H", [(1, 64), (700, 2048), (13, 8192), (66, 4160), (300, 448)])
@pytest.mark.parametrize("second,weighted", [(True, True), (False, False)])
def test_norm_is_rounded_to_the_nearest(moe, T, H, second, weighted):
    print(f"[case] norm {T} x {H} second={second} weighted={weighted}", flush=True)
    w = (1 + 0.3 * torch.randn(H, generator=torch.Generator().manual_seed(H))).to(torch.bfloat16) if weighted else None
    check_exact(moe, rows(T, H, T + 5), rows(T, H, T + 6) if second else None, w, 1e-6)


@pytest.mark.parametrize("exponent", [-120, -127, -129, -130, -133])
@pytest.mark.parametrize("weight", [None, 0, 20, 120, -60])
def test_norm_of_tiny_rows_without_eps(moe, exponent, weight):
    """1 / rms beyond the range of fp32, or its product with a weight, where the norm is an ordinary number"""
    print(f"[case] norm of rows of 2^{exponent}, weight 2^{weight}", flush=True)
    g = torch.Generator().manual_seed(3)
    x = (torch.randint(-7, 8, (9, 320), generator=g).double() * 2.0 ** exponent).to(torch.bfloat16)
    w = None if weight is None else ((1 + torch.rand(320, generator=g).double()) * 2.0 ** weight).to(torch.bfloat16)
    check_exact(moe, x, None, w, 0.0)


@pytest.mark.parametrize("exponent,weight", [(120, -110), (120, 100), (-60, 127), (100, -133)])
def test_norm_of_rows_and_weights_at_opposite_ends(moe, exponent, weight):
    print(f"[case] norm of rows of 2^{exponent}, weight 2^{weight}", flush=True)
    g = torch.Generator().manual_seed(4)
    x = (torch.randint(-7, 8, (9, 320), generator=g).double() * 2.0 ** exponent).to(torch.bfloat16)
    w = (torch.ones(320, dtype=torch.float64) * 2.0 ** weight).to(torch.bfloat16)
    check_exact(moe, x, None, w, 0.0)


def test_norm_with_weights_that_are_not_finite(moe):
    x, w = rows(5, 192, 8), torch.ones(192, dtype=torch.bfloat16)
    x[2, 3] = 0.0
    w[3], w[70], w[100] = float("inf"), float("-inf"), float("nan")
    _, out, q, scales = moe.moe_residual_norm_mx(x.cuda(), None, w.cuda())
    _, n = ref.norm(x, None, w, 1e-6)
    want = n.float().to(torch.bfloat16)
    out, qb, sb = out.cpu(), q.cpu().view(torch.uint8), scales.cpu().view(torch.uint8)
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and bool(torch.isnan(out[2, 3])) and bool(torch.isinf(out[:, 70]).all())
    special = ~torch.isfinite(n)
    assert torch.equal(out[special & ~torch.isnan(want)], want[special & ~torch.isnan(want)])
    bad = special.reshape(5, 6, 32).any(-1)
    assert torch.equal(sb == 255, bad) and bool((qb.reshape(5, 6, 32)[bad] == 0x7F).all())
