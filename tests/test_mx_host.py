"""The 8-bit layer's calls without a GPU: what they refuse (nothing is launched on these paths), workspace sizes, and the
64-bit reference that the GPU tests compare with, against torch's own 8-bit conversion."""
import ctypes

import pytest
import torch

from tests import mx_reference as ref

NULL, SHAPE, WS = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    import paper_2604_26881_amd as moe
    return moe.load()


p = ctypes.c_void_p(0x1000)      # never dereferenced
odd = ctypes.c_void_p(0x1008)    # not a multiple of 16
one = ctypes.c_void_p(0x1001)


def test_quantize_refusals(lib):
    call = lambda x=p, rows=4, H=64, q=p, s=p: lib.moe_quantize_mx(x, rows, H, q, s, None)
    assert call(rows=-1) == SHAPE and call(H=0) == SHAPE and call(H=96) == SHAPE
    assert call(x=None) == NULL and call(q=None) == NULL and call(s=None) == NULL
    assert call(x=odd) == SHAPE and call(q=odd) == SHAPE and call(s=one) == SHAPE
    assert call(x=None, rows=0, q=None, s=None) == 0


def test_norm_refusals(lib):
    def call(x=p, y=p, w=p, T=4, H=64, eps=1e-6, sum=p, out=p, q=p, s=p):
        return lib.moe_residual_norm_mx(x, y, w, T, H, ctypes.c_float(eps), sum, out, q, s, None)
    assert call(T=-1) == SHAPE and call(H=32) == SHAPE and call(H=8256) == SHAPE
    assert call(eps=-1.0) == SHAPE and call(eps=float("nan")) == SHAPE
    assert call(x=None) == NULL
    assert call(q=None) == NULL and call(s=None) == NULL          # both or neither
    assert call(sum=None, out=None, q=None, s=None) == NULL       # nothing wanted
    for name in ("x", "y", "w", "sum", "out", "q"):
        assert call(**{name: odd}) == SHAPE, name
    assert call(s=one) == SHAPE
    assert call(x=None, T=0) == 0


def test_route_refusals(lib):
    def call(x=p, Wr=p, b=p, T=4, H=64, E=16, K=2, score=0, G=1, top=1, best=1, renorm=0, scale=1.0, ids=p, w=p):
        return lib.moe_route_scored(x, Wr, b, T, H, E, K, score, G, top, best, renorm, ctypes.c_float(scale), ids, w, None)
    for bad in (dict(T=-1), dict(H=63), dict(H=8256), dict(E=0), dict(E=257), dict(K=0), dict(K=17, E=64), dict(K=5, E=4), dict(score=2),
                dict(score=-1), dict(G=0), dict(G=3), dict(E=256, G=128, top=128), dict(G=4, top=0), dict(G=4, top=5),
                dict(G=4, top=1, K=5), dict(best=0), dict(best=3), dict(G=16, top=16, best=2), dict(scale=float("inf")),
                dict(scale=float("nan")), dict(x=odd), dict(Wr=odd)):
        assert call(**bad) == SHAPE, bad
    for name in ("x", "Wr", "ids", "w"):
        assert call(**{name: None}) == NULL, name
    assert call(x=None, Wr=None, b=None, T=0, ids=None, w=None) == 0


def test_expert_block_refusals(lib):
    def call(lo=0, hi=8, x=p, xs=p, src=p, K=2, off=p, w=(p,) * 6, P=32, H=64, E=8, I=128, Y=p, ws=p, n=1 << 20):
        return lib.moe_expert_group_forward_mx(lo, hi, x, xs, src, K, off, *w, P, H, E, I, Y, ws, n, None)
    for bad in (dict(lo=3, hi=3), dict(lo=-1), dict(hi=9), dict(P=-1), dict(H=96), dict(I=32), dict(H=16448), dict(I=16448), dict(E=0, hi=0),
                dict(E=257), dict(K=0), dict(K=17), dict(K=3), dict(P=1 << 24, H=128), dict(x=odd), dict(Y=odd), dict(ws=odd), dict(xs=one)):
        assert call(**bad) == SHAPE, bad
    for name in ("x", "xs", "off", "Y", "ws"):
        assert call(**{name: None}) == NULL, name
    for i in range(6):
        assert call(w=tuple(None if j == i else p for j in range(6))) == NULL, i
        assert call(w=tuple(odd if j == i else p for j in range(6))) == SHAPE, i
    assert call(n=lib.moe_expert_workspace_bytes(32, 128) - 1) == WS
    assert call(x=None, P=0) == 0


def test_binding_refuses_before_it_looks_at_a_gpu():
    import paper_2604_26881_amd as moe
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(moe.MoeError, match="multiple of 64"):
        moe.moe_quantize_mx(x[:, :32])
    with pytest.raises(moe.MoeError, match="multiple of 64"):
        moe.moe_residual_norm_mx(x[:, :32])
    with pytest.raises(moe.MoeError, match="score must be"):
        moe.moe_route_scored(x, x, None, 2, score="relu")
    pair = lambda *s: (torch.zeros(s, dtype=torch.uint8).view(torch.float8_e4m3fn),
                       torch.zeros((*s[:-1], s[-1] // 32), dtype=torch.uint8).view(torch.float8_e8m0fnu))
    W, off, Y, src = pair(2, 64, 64), torch.zeros(3, dtype=torch.int32), torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    block = lambda src=None, K=1, off=off: moe.moe_expert_group_forward_mx(0, 2, pair(4, 64), src, K, off, W, W, W, Y)
    with pytest.raises(moe.MoeError, match="P / K rows"):
        block(src=src, K=2)
    with pytest.raises(moe.MoeError, match="E . 1 entries"):
        block(off=off[:2])
    for call in (lambda: moe.moe_quantize_mx(x), lambda: moe.moe_residual_norm_mx(x), lambda: moe.moe_route_scored(x, x, None, 2), block):
        with pytest.raises(moe.MoeError, match="on the current GPU"):
            call()


def test_reference_conversion_is_torchs_where_nothing_saturates():
    g = torch.Generator().manual_seed(3)
    t = torch.cat([torch.randn(4096, generator=g) * 100, torch.randn(4096, generator=g) * 0.01, torch.tensor([448.0, -448.0, 0.0, 2.0 ** -9, 2.0 ** -10])])
    t = t.clamp(-448, 448)
    assert torch.equal(ref.to_e4m3(t.double()), t.to(torch.float8_e4m3fn).double())
    # the scale: largest magnitude at most 448 of it, and more than 224 of it (it is the smallest one)
    v = torch.randn(64, 256, generator=g).double() * torch.exp(3 * torch.randn(64, 1, generator=g).double())
    top, scale = v.reshape(64, 8, 32).abs().amax(-1), ref.two_to(ref.block_exponent(v))
    assert bool((top <= 448 * scale).all()) and bool((top > 224 * scale).all())
    assert ref.block_exponent(torch.full((1, 32), 448.0, dtype=torch.float64)).item() == 0
    assert ref.block_exponent(torch.full((1, 32), 448.0001, dtype=torch.float64)).item() == 1
    assert ref.block_exponent(torch.zeros(1, 32, dtype=torch.float64)).item() == -126
    q, _ = ref.mx(v)
    assert bool(((q - v).abs() <= 2.0 ** -4 * v.abs() + 2.0 ** -10 * scale.repeat_interleave(32, -1)).all())
