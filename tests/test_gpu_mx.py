"""The 8-bit layer's calls on the GPU against their definitions in 64 bits (mx_reference.py).

Tolerances.  Conversion of bf16 rows: to the bit (the scale follows from bits, the quotient is exact, one rounding).  Norm: a
sum of squares of up to 8192 values is at most 42 fp32 roundings long (32 per lane, 8 joins, 2), half of that after the root,
and six more steps: 2^-19 of the value covers it; bf16 rounds by 2^-8 at most, e4m3 by 2^-4 of the value or, below its normal
range, half of 2^-9 * scale.  Gating: ids equal; weights: logits are fp32 sums in some order, off by at most 32 * 2^-24
(beyond H 2048 H / 64 * 2^-24) of |x[t]| * max |Wr[e]| (a step of 32 products by 6 * 2^-24 of its terms' magnitudes), which moves a softmax or sigmoid by at most
twice that of its value and a renormalised one by twice that again; sum, quotient and product 2^-20.  Expert rows: element by element what mx_reference.experts bounds; and, much closer, the 2-norm
over a row: two roundings to bf16 (of the hidden row, of the output), each uniform within 2^-8 at most, are 2^-8 / sqrt(3) in
the mean square or less, together 3.2e-3; the matrix instruction's own cuts 1e-4.  A row's 64 to 16384 elements scatter around
that: twice it is allowed for a row, and it for a batch of 2048 elements and more."""
import pytest
import torch

from tests import mx_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    import paper_2604_26881_amd as m
    assert torch.cuda.is_available(), "these tests need the GPU"
    m.load()
    return m


def bits(t):
    return t.view(torch.int16 if t.element_size() == 2 else torch.uint8)


def rows(T, H, seed, spread=0.7):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((T, H), generator=g) * torch.exp(spread * torch.randn(H, generator=g))).to(torch.bfloat16)


# ---- conversion

@pytest.mark.parametrize("n,H", [(1, 64), (3, 192), (13, 2048), (1, 16384), (1000, 320), (257, 1408)])
def test_quantize_is_the_definition_to_the_bit(moe, n, H):
    print(f"[case] quantize {n} x {H}", flush=True)
    x = rows(n, H, n + H, 2.0)
    q, s = moe.moe_quantize_mx(x.cuda())
    want, e = ref.mx(x.double())
    assert torch.equal(s.cpu().view(torch.uint8).int(), (e + 127).int())
    assert torch.equal(ref.values((q, s)), want)


def test_quantize_of_extreme_blocks(moe):
    x = torch.zeros(12, 64)
    x[1, 3] = 2.0 ** -133                  # a subnormal: the smallest scale
    x[2, 5] = float(torch.finfo(torch.bfloat16).max)
    x[3, 7], x[3, 40] = float("inf"), 1.0
    x[4, 9], x[4, 41] = float("nan"), -2.0
    x[5, 0] = float("-inf")
    x[6] = 448.0
    x[7] = 450.0                           # one bf16 above: the next scale
    x[8, :32], x[8, 32:] = 1.0, 2.0 ** -100
    x[9, 0], x[9, 1:32] = 448.0, 2.0 ** -10       # half of the smallest value of this scale: to even, zero
    x[10, 0], x[10, 1:32] = 448.0, 1.5 * 2.0 ** -9
    x[11, 31] = -0.0
    x = x.to(torch.bfloat16)
    q, s = moe.moe_quantize_mx(x.cuda())
    v, sb, qb = ref.values((q, s)), s.cpu().view(torch.uint8), q.cpu().view(torch.uint8)
    want, e = ref.mx(torch.nan_to_num(x.double(), nan=0.0, posinf=0.0, neginf=0.0))
    bad = ~torch.isfinite(x.reshape(12, 2, 32)).all(-1)
    assert torch.equal(sb[~bad].int(), (e + 127).int()[~bad]) and bool((sb[bad] == 255).all())
    assert bool((qb.reshape(12, 2, 32)[bad] == 0x7F).all())
    ok = ~bad.repeat_interleave(32, 1)
    assert torch.equal(v[ok], want[ok])


# ---- norm

def check_norm(moe, x, y, w, eps=1e-6, **kw):
    got = moe.moe_residual_norm_mx(x.cuda(), None if y is None else y.cuda(), None if w is None else w.cuda(), eps, **kw)
    u, n = ref.norm(x, y, w, eps)
    f32 = 2.0 ** -19
    if got[0] is not None:
        assert bool(((got[0].cpu().double() - u).abs() <= (2.0 ** -8 + 2.0 ** -23) * u.abs()).all())
    if got[1] is not None:
        assert bool(((got[1].cpu().double() - n).abs() <= (2.0 ** -8 + f32) * n.abs()).all())
    if got[2] is not None:
        v, scale = ref.values(got[2:]), got[3].cpu().double()
        s = scale.repeat_interleave(32, -1)
        assert bool(((v - n).abs() <= (2.0 ** -4 + 2 * f32) * n.abs() + 2.0 ** -10 * s).all())
        top = n.reshape(*scale.shape, 32).abs().amax(-1)
        assert bool((top <= 448 * scale * (1 + f32)).all())
        assert bool(((top >= 224 * scale * (1 - f32)) | (scale == 2.0 ** -126)).all())
    return got


@pytest.mark.parametrize("T,H", [(1, 64), (5, 192), (1, 2048), (3, 8192), (777, 2048), (66, 4160), (300, 448)])
@pytest.mark.parametrize("second,weighted", [(True, True), (False, False), (True, False), (False, True)])
def test_norm_every_element(moe, T, H, second, weighted):
    print(f"[case] norm {T} x {H} second={second} weighted={weighted}", flush=True)
    x, y = rows(T, H, T), rows(T, H, T + 1) if second else None
    w = (1 + 0.3 * torch.randn(H, generator=torch.Generator().manual_seed(H))).to(torch.bfloat16) if weighted else None
    full = check_norm(moe, x, y, w)
    # a result does not depend on which others are asked for
    for keep in ((True, False, False), (False, True, False), (False, False, True), (True, False, True)):
        some = moe.moe_residual_norm_mx(x.cuda(), None if y is None else y.cuda(), None if w is None else w.cuda(), keep_sum=keep[0],
                                        keep_out=keep[1], quantize=keep[2])
        for a, b, k in zip(some, full, (keep[0], keep[1], keep[2], keep[2])):
            assert (a is None) == (not k) and (a is None or torch.equal(bits(a), bits(b)))


def test_norm_in_place_and_rows_of_zeros_and_nan(moe):
    T, H = 9, 512
    x, y = rows(T, H, 1), rows(T, H, 2)
    x[3], y[3] = 0, 0                                   # a padded row: zeros, whatever eps
    want = moe.moe_residual_norm_mx(x.cuda(), y.cuda())
    assert not bool(want[1][3].float().any()) and not bool(want[2][3].float().any())
    xg, yg = x.cuda(), y.cuda()
    got = moe.moe_residual_norm_mx(xg, yg, sum=yg, out=xg)
    assert got[0] is yg and got[1] is xg
    for a, b in zip(got, want):
        assert torch.equal(bits(a), bits(b))
    x[5, 17] = float("nan")
    x[6, 200] = float("inf")
    bad = moe.moe_residual_norm_mx(x.cuda(), y.cuda())
    for a, b in zip(bad, want):                         # other rows: untouched
        keep = [t for t in range(T) if t not in (5, 6)]
        assert torch.equal(bits(a[keep]), bits(b[keep]))
    assert bool(torch.isnan(bad[1][5]).all()) and bool(torch.isnan(bad[2][5].float()).all()) and bool((bad[3][5].view(torch.uint8) == 255).all())
    v = bad[2][6].float()
    assert bool(torch.isnan(v[192:224]).all()) and not bool(torch.isnan(v[:192]).any()) and not bool(torch.isnan(v[224:]).any())


@pytest.mark.parametrize("exponent,eps", [(100, 1e-6), (118, 0.0), (-40, 0.0), (-100, 0.0), (-100, 1e-6)])
def test_norm_of_rows_whose_squares_leave_fp32(moe, exponent, eps):
    x = (rows(9, 320, 17).double() * 2.0 ** exponent).to(torch.bfloat16)
    y = (rows(9, 320, 18).double() * 2.0 ** exponent).to(torch.bfloat16)
    check_norm(moe, x, y, rows(1, 320, 19)[0], eps)


# ---- gating

ROUTE = [  # T, H, E, K, score, groups, top_groups, best, renorm, scale, balance
    (1, 64, 8, 2, "softmax", 1, 1, 1, False, 1.0, False),
    (13, 2048, 60, 4, "softmax", 1, 1, 1, False, 1.0, False),
    (37, 192, 256, 8, "sigmoid", 8, 4, 2, True, 2.5, True),
    (40, 1088, 256, 16, "sigmoid", 1, 1, 1, True, 1.0, True),
    (19, 512, 96, 6, "softmax", 4, 2, 1, True, 1.0, True),
    (9, 4096, 160, 6, "softmax", 8, 3, 1, False, 16.0, False),
    (7, 8192, 64, 8, "sigmoid", 64, 8, 1, True, 1.0, True),
    (300, 320, 17, 3, "sigmoid", 1, 1, 1, False, 0.5, True),
    (5, 128, 1, 1, "softmax", 1, 1, 1, True, 1.0, False),
    (70, 640, 200, 10, "sigmoid", 5, 2, 2, True, 1.0, True),
]


def gate_inputs(T, H, E, seed, balance):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, H), generator=g).to(torch.bfloat16)
    Wr = (torch.randn((E, H), generator=g) * (1.0 / H ** 0.5)).to(torch.bfloat16)
    return x, Wr, torch.randn(E, generator=g) * balance if balance else None


def check_route(moe, x, Wr, b, K, score, G, top, best, renorm, scale):
    ids, w = moe.moe_route_scored(x.cuda(), Wr.cuda(), None if b is None else b.cuda(), K, score, G, top, best, renorm, scale)
    rid, rw = ref.route(x, Wr, b, K, score, G, top, best, renorm, scale)
    assert torch.equal(ids.cpu(), rid), (ids.cpu() != rid).nonzero()[:4]
    finite = torch.isfinite(rw)
    w = w.cpu().double()
    assert torch.equal(torch.isnan(w), torch.isnan(rw))
    doubt = max(32, x.shape[1] / 64) * 2.0 ** -24 * x.double().norm(dim=1, keepdim=True) * Wr.double().norm(dim=1).max()
    assert bool(((w - rw).abs() <= (4 * doubt + 2.0 ** -20) * rw.abs() + 1e-38)[finite].all())
    return ids, w


@pytest.mark.parametrize("case", ROUTE, ids=lambda c: "-".join(map(str, c[:5])))
def test_route_scored_chooses_like_the_definition(moe, case):
    T, H, E, K, score, G, top, best, renorm, scale, balance = case
    print(f"[case] route_scored {case}", flush=True)
    x, Wr, b = gate_inputs(T, H, E, T * 7 + H, (0.1 if score == "sigmoid" else 0.5 / E) if balance else 0.0)
    ids, w = check_route(moe, x, Wr, b, K, score, G, top, best, renorm, scale)
    assert bool((ids.sort(1).values.diff(dim=1) > 0).all())      # K different experts
    # a row depends on itself alone, to the bit
    for t in {0, T // 2, T - 1}:
        i1, w1 = moe.moe_route_scored(x[t:t + 1].cuda(), Wr.cuda(), None if b is None else b.cuda(), K, score, G, top, best, renorm, scale)
        assert torch.equal(i1[0], ids[t]) and torch.equal(w1[0].cpu().double(), w[t])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_scored_without_extras_chooses_like_moe_route(moe, score):
    x, Wr, _ = gate_inputs(500, 1024, 60, 5, 0)
    a, _ = moe.moe_route(x.cuda(), Wr.cuda(), None, 4, True)
    b, _ = moe.moe_route_scored(x.cuda(), Wr.cuda(), None, 4, score, renorm=True)
    assert torch.equal(a, b)


def test_route_scored_near_ties_and_exact_ties(moe):
    """Router rows that differ in their last bits: logits a few units apart, and equal ones, at every border of the choice."""
    T, H, E = 48, 1536, 64
    g = torch.Generator().manual_seed(11)
    x = torch.randn((T, H), generator=g).to(torch.bfloat16)
    base = (torch.randn((8, H), generator=g) * 0.02).to(torch.bfloat16)
    Wr = base.repeat(8, 1)                                    # expert e is base row e % 8: eight equal logits each
    near = Wr.view(torch.int16).clone()
    at = torch.randint(0, H, (E,), generator=g)
    near[torch.arange(E), at] += torch.randint(-1, 2, (E,), generator=g).to(torch.int16)     # one element off by a unit, or not at all
    perm = torch.randperm(H, generator=g)
    for W in (Wr, near.view(torch.bfloat16)):
        for args in ((6, "softmax", 1, 1, 1, True, 1.0), (8, "sigmoid", 8, 3, 2, True, 1.0), (4, "sigmoid", 4, 2, 1, False, 1.0)):
            print(f"[case] ties {args}", flush=True)
            check_route(moe, x, W, None, *args)
            check_route(moe, x, W, (torch.randint(-2, 3, (E,), generator=g).float() * 2.0 ** -24), *args)
    check_route(moe, x[:, perm], Wr[:, perm], None, 6, "softmax", 1, 1, 1, True, 1.0)
    check_route(moe, torch.zeros_like(x), Wr, None, 8, "sigmoid", 8, 3, 2, True, 1.0)        # padded rows: every expert ties


def test_route_scored_masks_and_values_that_are_not_finite(moe):
    T, H, E, K = 12, 256, 32, 4
    x, Wr, b = gate_inputs(T, H, E, 3, 0.1)
    inf = float("inf")
    for G, top, best in ((1, 1, 1), (4, 2, 2), (4, 2, 1)):
        masked = b.clone()
        masked[::3] = -inf                                     # experts that are off
        check_route(moe, x, Wr, masked, K, "sigmoid", G, top, best, True, 1.0)
        masked[:] = -inf                                       # all of them: the lowest ids
        check_route(moe, x, Wr, masked, K, "sigmoid", G, top, best, True, 1.0)
        masked[:] = torch.finfo(torch.float32).min             # the type's lowest value: a sum of two is -infinity
        check_route(moe, x, Wr, masked, K, "softmax", G, top, best, True, 1.0)
        masked = b.clone()
        masked[5], masked[9] = inf, float("nan")
        check_route(moe, x, Wr, masked, K, "sigmoid", G, top, best, True, 1.0)
    y = x.clone()
    y[3, 7], y[4, 8] = float("nan"), inf
    ids, w = check_route(moe, y, Wr, b, K, "sigmoid", 4, 2, 2, True, 1.0)
    ids, w = check_route(moe, y, Wr, None, K, "softmax", 1, 1, 1, True, 1.0)
    assert torch.equal(ids[3].cpu(), torch.arange(K, dtype=torch.int32)) and bool(torch.isnan(w[3]).all())
    # scores that underflow: weights are 0, not 0 / 0
    deep = torch.zeros(T, H, dtype=torch.bfloat16)
    deep[:, 0] = 1.0
    W0 = torch.zeros(E, H, dtype=torch.bfloat16)
    W0[:, 0] = -1000.0
    _, w = moe.moe_route_scored(deep.cuda(), W0.cuda(), None, K, "sigmoid", renorm=True)
    assert not bool(w.any())


# ---- expert blocks

def block_case(moe, counts, H, I, seed, std=None):
    E, P = len(counts), sum(counts)
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((P, H), generator=g) * torch.exp(0.7 * torch.randn(H, generator=g))).to(torch.bfloat16).cuda()
    w = [(torch.randn((E, n, k), generator=g) * (std or 0.7 / k ** 0.5)).to(torch.bfloat16).cuda() for n, k in ((I, H), (I, H), (H, I))]
    c = dict(E=E, P=P, H=H, I=I, counts=list(counts), x=moe.moe_quantize_mx(x), Wg=moe.moe_quantize_mx(w[0]), Wu=moe.moe_quantize_mx(w[1]),
             Wd=moe.moe_quantize_mx(w[2]), off=torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32).cuda())
    return c


def run_block(moe, c, cuts=None, src=None, K=1, x=None, Yp=None):
    Yp = torch.full((c["P"], c["H"]), 768.0, dtype=torch.bfloat16, device="cuda") if Yp is None else Yp
    for lo, hi in cuts or [(0, c["E"])]:
        moe.moe_expert_group_forward_mx(lo, hi, c["x"] if x is None else x, src, K, c["off"], c["Wg"], c["Wu"], c["Wd"], Yp)
    torch.cuda.synchronize()
    return Yp


def check_block(c, Yp):
    Y, tol = ref.experts(ref.values(c["x"]), torch.arange(c["P"]), c["counts"], ref.values(c["Wg"]), ref.values(c["Wu"]), ref.values(c["Wd"]))
    d = (Yp.cpu().double() - Y).abs()
    assert bool((d <= tol).all()), f"{int((d > tol).sum())} of {d.numel()} elements, worst {float((d / tol).max()):.3g} of the tolerance at {(d / tol).argmax()}"
    rel = d.norm(dim=1) / Y.norm(dim=1).clamp_min(1e-30)
    assert float(rel.max()) <= 6.6e-3, (float(rel.max()), int(rel.argmax()))
    if d.numel() >= 2048:
        assert float(d.norm() / Y.norm()) <= 3.3e-3, float(d.norm() / Y.norm())


COUNTS = [  # rows per expert (names the kernels by their mean), H, I
    ([1], 64, 64), ([1, 0, 0, 2], 64, 128), ([0, 3, 1, 0, 16, 17, 5, 2], 192, 320), ([1, 2, 1, 0, 4], 2048, 1408), ([15, 16, 17, 33, 0, 1], 448, 576),
    ([31, 32, 33, 64, 65, 1], 256, 192), ([40, 63, 100, 129, 1, 0, 7], 320, 448), ([128, 127, 300, 1, 0, 255, 256, 257], 512, 384),
    ([100, 60, 128, 129, 0, 65, 200, 31], 384, 320), ([100, 60, 128, 129, 0, 65, 200, 31], 448, 192), ([33, 40, 64, 63, 65, 1, 0, 50], 256, 256),
    ([700, 90], 1088, 704), ([513], 192, 256), ([2, 3], 16384, 64), ([3, 2], 64, 16384),
]


@pytest.mark.parametrize("counts,H,I", COUNTS, ids=lambda v: str(v).replace(" ", "") if isinstance(v, list) else str(v))
def test_expert_rows_every_element(moe, counts, H, I):
    print(f"[case] experts mx counts={counts} H={H} I={I}", flush=True)
    c = block_case(moe, counts, H, I, H + I + len(counts))
    Yp = run_block(moe, c)
    check_block(c, Yp)
    # the same bits whatever the block cut, and only the rows of the experts asked for are written
    if c["E"] > 2:
        cuts = [(2, c["E"]), (0, 1), (1, 2)]
        assert torch.equal(bits(run_block(moe, c, cuts)), bits(Yp))
        part = run_block(moe, c, [(1, 2)])
        lo, hi = sum(counts[:1]), sum(counts[:2])
        assert torch.equal(bits(part[lo:hi]), bits(Yp[lo:hi])) and bool((part[:lo] == 768).all()) and bool((part[hi:] == 768).all())


@pytest.mark.parametrize("T,H,E,K,I", [(1, 128, 8, 2, 64), (33, 320, 16, 4, 192), (200, 512, 12, 3, 448), (700, 256, 4, 2, 320), (1500, 512, 20, 2, 2048)])
def test_rows_read_through_the_sort_equal_the_permuted_copy(moe, T, H, E, K, I):
    print(f"[case] gather T={T} H={H} E={E} K={K} I={I}", flush=True)
    g = torch.Generator().manual_seed(T)
    ids = torch.rand((T, E), generator=g).argsort(1)[:, :K].to(torch.int32).cuda().contiguous()
    x = rows(T, H, T).cuda()
    off, src, _, _ = moe.moe_permute(ids, x, E, materialize=False)
    counts = off.cpu().diff().tolist()
    c = block_case(moe, counts, H, I, T + 1)
    q = moe.moe_quantize_mx(x)
    at = (src // K).long()
    c["x"] = tuple(t.view(torch.uint8)[at].view(t.dtype) for t in q)
    Yp = run_block(moe, c)
    check_block(c, Yp)
    assert torch.equal(bits(run_block(moe, c, src=src, K=K, x=q)), bits(Yp))


def test_experts_without_rows_are_not_read_and_nan_stays_in_its_row(moe):
    for counts in ([3, 0, 5, 0], [200, 0, 90, 0]):
        c = block_case(moe, counts, 256, 192, 9)
        want = run_block(moe, c)
        for e in (1, 3):                         # NaN weights and scales of experts nobody chose
            for w in ("Wg", "Wu", "Wd"):
                for t in c[w]:
                    t.view(torch.uint8)[e] = 255
        assert torch.equal(bits(run_block(moe, c)), bits(want))
        c["x"][1].view(torch.uint8)[1, 3] = 255  # one block of one row
        got = run_block(moe, c)
        keep = [r for r in range(c["P"]) if r != 1]
        assert bool(torch.isnan(got[1]).all()) and torch.equal(bits(got[keep]), bits(want[keep]))


def test_scales_far_apart_and_zero_rows(moe):
    c = block_case(moe, [20, 70, 1], 256, 128, 4)
    g = torch.Generator().manual_seed(5)
    s = c["x"][1].view(torch.uint8)
    s[:] = (s.int() + torch.randint(-20, 6, s.shape, generator=g).cuda()).clamp(1, 250).to(torch.uint8)
    for w in ("Wg", "Wu", "Wd"):
        s = c[w][1].view(torch.uint8)
        s[:] = (s.int() + torch.randint(-12, 3, s.shape, generator=g).cuda()).clamp(1, 250).to(torch.uint8)
    c["x"][0].view(torch.uint8)[7] = 0           # a row of zeros
    c["x"][1].view(torch.uint8)[8] = 1           # a row of the smallest scale: products that vanish
    Yp = run_block(moe, c)
    check_block(c, Yp)
    assert not bool(Yp[7].float().any())


def test_binding_refuses_tensors_of_another_shape_type_layout_or_device(moe):
    x = rows(4, 128, 1).cuda()
    bad = lambda match, call: _refused(moe, match, call)
    q, s = moe.moe_quantize_mx(x)
    bad("x must be contiguous", lambda: moe.moe_quantize_mx(torch.zeros((64, 64), dtype=torch.bfloat16, device="cuda").t()))
    bad("x must be torch.bfloat16", lambda: moe.moe_quantize_mx(x.float()))
    bad("q must be", lambda: moe.moe_quantize_mx(x, q=q[:2]))
    bad("scales must be", lambda: moe.moe_quantize_mx(x, scales=s.view(torch.uint8)))
    bad("y must be", lambda: moe.moe_residual_norm_mx(x, x[:2]))
    bad("weight must be", lambda: moe.moe_residual_norm_mx(x, None, x[0, :64]))
    bad("weight must be on the current GPU", lambda: moe.moe_residual_norm_mx(x, None, x[0].cpu()))
    bad("sum must be", lambda: moe.moe_residual_norm_mx(x, sum=x[:, :64].contiguous()))
    bad("Wr must be", lambda: moe.moe_route_scored(x, x[:, :64].contiguous(), None, 2))
    bad("balance must be", lambda: moe.moe_route_scored(x, x, torch.zeros(5).cuda(), 2))
    bad("topk_ids must be", lambda: moe.moe_route_scored(x, x, None, 2, topk_ids=torch.zeros(4, 2).cuda()))
    c = block_case(moe, [2, 2], 128, 64, 1)
    run = lambda **kw: run_block(moe, dict(c, **kw))
    bad("x must be", lambda: run(x=moe.moe_quantize_mx(x[:3].contiguous())))
    bad("x scales must be", lambda: run(x=(c["x"][0], c["x"][1][:, :2].contiguous())))
    bad("Wu must be", lambda: run(Wu=c["Wd"]))
    bad("Wd scales must be", lambda: run(Wd=(c["Wd"][0], c["Wu"][1])))
    bad("Yp must be", lambda: run_block(moe, c, Yp=torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")))
    bad("workspace too small", lambda: moe.moe_expert_group_forward_mx(0, 2, c["x"], None, 1, c["off"], c["Wg"], c["Wu"], c["Wd"], run_block(moe, c),
                                                                       torch.zeros(16, dtype=torch.uint8, device="cuda")))


def _refused(moe, match, call):
    with pytest.raises(moe.MoeError, match=match):
        call()


# ---- together, as a serving loop uses them

def layer(moe, s):
    moe.moe_residual_norm_mx(s["x"], s["y"], s["w"], 1e-6, sum=s["sum"], out=s["out"], q=s["q"], scales=s["scales"])
    moe.moe_route_scored(s["out"], s["Wr"], s["b"], s["K"], "sigmoid", 4, 2, 2, True, 2.5, s["ids"], s["tw"])
    moe.moe_permute(s["ids"], s["out"], s["E"], s["off"], s["src"], s["row"], None, s["pws"], materialize=False)
    for lo, hi in ((0, 5), (5, s["E"])):
        moe.moe_expert_group_forward_mx(lo, hi, (s["q"], s["scales"]), s["src"], s["K"], s["off"], s["Wg"], s["Wu"], s["Wd"], s["Yp"], s["ws"])
    moe.moe_combine(s["Yp"], s["row"], s["tw"], None, None, s["res"])


def layer_state(moe, T, H, E, K, I, seed):
    g = torch.Generator().manual_seed(seed)
    P, dev = T * K, "cuda"
    w = [(torch.randn((E, n, k), generator=g) * 0.05).to(torch.bfloat16).to(dev) for n, k in ((I, H), (I, H), (H, I))]
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32, device=dev)
    bf = lambda *n: torch.zeros(n, dtype=torch.bfloat16, device=dev)
    q, scales = moe.moe_quantize_mx(bf(T, H))
    return dict(T=T, H=H, E=E, K=K, I=I, P=P, x=rows(T, H, seed).to(dev), y=rows(T, H, seed + 1).to(dev),
                w=(1 + 0.2 * torch.randn(H, generator=g)).to(torch.bfloat16).to(dev), Wr=(torch.randn((E, H), generator=g) * 0.05).to(torch.bfloat16).to(dev),
                b=(torch.randn(E, generator=g) * 0.05).to(dev), Wg=moe.moe_quantize_mx(w[0]), Wu=moe.moe_quantize_mx(w[1]), Wd=moe.moe_quantize_mx(w[2]),
                sum=bf(T, H), out=bf(T, H), q=q, scales=scales, ids=i32(T, K), tw=torch.zeros((T, K), device=dev), off=i32(E + 1), src=i32(P), row=i32(P),
                pws=torch.zeros(max(int(moe.load().moe_permute_workspace_bytes(T, K, E)), 256), dtype=torch.uint8, device=dev), Yp=bf(P, H), res=bf(T, H),
                ws=torch.zeros(int(moe.load().moe_expert_workspace_bytes(P, I)), dtype=torch.uint8, device=dev))


@pytest.mark.parametrize("T", [1, 37, 900])
def test_layer_in_8_bits(moe, T):
    print(f"[case] layer in 8 bits T={T}", flush=True)
    s = layer_state(moe, T, 512, 16, 4, 320, T)
    layer(moe, s)
    torch.cuda.synchronize()
    # every step against its definition, on the inputs that it had
    check_norm(moe, s["x"].cpu(), s["y"].cpu(), s["w"].cpu())
    check_route(moe, s["out"].cpu(), s["Wr"].cpu(), s["b"].cpu(), 4, "sigmoid", 4, 2, 2, True, 2.5)
    c = dict(s, counts=s["off"].cpu().diff().tolist())
    at = (s["src"] // s["K"]).long()
    c["x"] = tuple(t.view(torch.uint8)[at].view(t.dtype) for t in (s["q"], s["scales"]))
    check_block(c, s["Yp"])
    Yp, row, tw = s["Yp"].cpu().double(), s["row"].cpu().long().reshape(T, 4), s["tw"].cpu().double()
    want = (Yp[row] * tw[..., None]).sum(1)
    d = (s["res"].cpu().double() - want).abs()
    assert bool((d <= 2.0 ** -8 * want.abs() + 8 * 2.0 ** -24 * (Yp[row].abs() * tw[..., None].abs()).sum(1) + 1e-30).all())


@pytest.mark.parametrize("T,H,I", [(1, 512, 320), (150, 256, 192), (300, 1024, 1600)])     # streamed, and in tiles
def test_captured_layer_replays_like_the_eager_one_on_another_stream(moe, T, H, I):
    s = layer_state(moe, T, H, 16, 4, I, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(moe, s)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(moe, s)
    for k in range(4):
        s["x"].copy_(rows(T, H, 50 + k).cuda())
        layer(moe, s)
        torch.cuda.synchronize()
        want = {n: s[n].clone() for n in ("sum", "out", "ids", "Yp", "res")}
        for n in want:
            s[n].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(s[n].view(torch.uint8), want[n].view(torch.uint8)), (k, n)


def test_batches_of_no_tokens(moe):
    s = layer_state(moe, 2, 128, 8, 2, 64, 1)
    none = lambda t: t[:0]
    a = moe.moe_residual_norm_mx(none(s["x"]), none(s["y"]), s["w"])
    assert [tuple(t.shape) for t in a] == [(0, 128), (0, 128), (0, 128), (0, 4)]
    ids, w = moe.moe_route_scored(none(s["x"]), s["Wr"], s["b"], 2)
    assert ids.shape == (0, 2) and w.shape == (0, 2)
    off = torch.zeros(9, dtype=torch.int32, device="cuda")
    y = moe.moe_expert_group_forward_mx(0, 8, a[2:], torch.zeros(0, dtype=torch.int32, device="cuda"), 2, off, s["Wg"], s["Wu"], s["Wd"], none(s["Yp"]))
    assert y.shape == (0, 128)
    assert moe.moe_quantize_mx(none(s["x"]))[0].shape == (0, 128)


# ---- the ends of the ranges

BATCHES = [  # H, E, K, score, groups, top_groups, best, renorm, scale, balance
    (192, 60, 4, "softmax", 1, 1, 1, False, 1.0, False),
    (128, 256, 8, "softmax", 8, 3, 2, True, 1.0, True),
    (128, 176, 6, "softmax", 1, 1, 1, False, 1.0, True),
    (256, 96, 16, "sigmoid", 16, 4, 2, True, 2.5, True),
]


@pytest.mark.parametrize("case", BATCHES, ids=lambda c: "-".join(map(str, c[:5])))
def test_route_scored_rows_are_the_same_in_batches_of_every_size(moe, case):
    H, E, K, score, groups, top, best, renorm, scale, balance = case
    T = 5003
    print(f"[case] route_scored batches {case}", flush=True)
    x, Wr, b = gate_inputs(T, H, E, H + E, (0.1 if score == "sigmoid" else 0.5 / E) if balance else 0.0)
    x[::7] = x[3]                                              # (and equal rows are equal wherever they stand)
    run = lambda rows: moe.moe_route_scored(rows.cuda(), Wr.cuda(), None if b is None else b.cuda(), K, score, groups, top, best, renorm, scale)
    ids, w = run(x)
    assert torch.equal(w[::7], w[3:4].expand(len(w[::7]), K)) and torch.equal(ids[::7], ids[3:4].expand(len(ids[::7]), K))
    for lo, hi in ((0, 300), (4990, T), (2500, 2501)):
        some_ids, some_w = run(x[lo:hi].contiguous())
        assert torch.equal(some_ids, ids[lo:hi]) and torch.equal(some_w.view(torch.int32), w[lo:hi].view(torch.int32))
    check_route(moe, x[:40], Wr, b, K, score, groups, top, best, renorm, scale)


@pytest.mark.parametrize("T,H,E,K,score,groups,top,best", [(4200, 64, 20, 3, "softmax", 1, 1, 1), (4100, 128, 64, 16, "sigmoid", 16, 5, 2),
                                                           (33, 128, 256, 16, "sigmoid", 64, 32, 2), (20, 192, 129, 16, "softmax", 43, 6, 1)])
def test_route_scored_large_batches_and_many_groups(moe, T, H, E, K, score, groups, top, best):
    print(f"[case] route_scored {T} {H} {E} {K} {score} {groups}", flush=True)
    x, Wr, b = gate_inputs(T, H, E, T, 0.1 if score == "sigmoid" else 0.5 / E)
    check_route(moe, x, Wr, b, K, score, groups, top, best, True, 1.0)


HEIGHTS = [300, 64, 65, 1, 0, 128, 192, 256, 257, 30, 90, 500, 20, 33, 127, 250, 5, 70, 64, 10]
MORE_COUNTS = [  # mean rows of 13 to 24 (two tiles of 16), above 24, and hundreds; scale rows of odd numbers of pairs and of part groups
    ([24, 24, 13, 30, 2, 0], 704, 832), ([33, 15, 1, 17, 32, 31, 0, 16], 2048, 1408), ([40, 63, 100, 129, 1, 0, 7], 576, 704),
    ([40, 63, 100, 129, 1, 0, 7], 640, 576), ([300, 280, 260, 0], 1152, 1216), ([129, 200, 33, 0, 256, 257], 1600, 512), ([26], 4160, 2112),
    # more workgroups than compute units, few rows each: one row, pieces of 4 and 8 rows that are full, begun or two
    ([1] * 64, 512, 576), ([1, 0, 3, 4, 5, 8, 9, 16, 17, 12, 2, 7, 0, 13, 20, 33, 6, 1, 15, 10, 11, 14, 3, 8], 1088, 704), ([4, 8, 5, 1] * 10, 1024, 1408),
    # tiles of every height, more than workgroups: several rounds of the walk, of gate/up and of down
    (HEIGHTS, 512, 4096), (HEIGHTS, 4096, 576), (HEIGHTS, 3648, 1088),
    ([40], 16384, 576), ([70, 3], 576, 16384),                 # the longest contractions in tiles
]


@pytest.mark.parametrize("counts,H,I", MORE_COUNTS, ids=lambda v: str(v).replace(" ", "") if isinstance(v, list) else str(v))
def test_expert_rows_of_more_sizes(moe, counts, H, I):
    print(f"[case] experts mx counts={counts} H={H} I={I}", flush=True)
    c = block_case(moe, counts, H, I, H + I + len(counts))
    Yp = run_block(moe, c)
    check_block(c, Yp)
    # scales of the rows may lie at any even address
    n = c["x"][1].numel()
    room = torch.zeros(n + 16, dtype=torch.uint8, device="cuda")
    for at in (2, 6):
        room[at:at + n] = c["x"][1].view(torch.uint8).reshape(-1)
        shifted = room[at:at + n].view(torch.float8_e8m0fnu).view(c["P"], H // 32)
        assert shifted.data_ptr() % 4 == 2
        assert torch.equal(bits(run_block(moe, dict(c, x=(c["x"][0], shifted)))), bits(Yp))


def test_two_blocks_at_once_share_a_workspace(moe):
    for counts in ([9, 3, 12, 8, 1, 7], [90, 30, 120, 80, 10, 70]):
        c = block_case(moe, counts, 512, 640, 6)
        want = run_block(moe, c)
        ws = torch.empty(int(moe.load().moe_expert_workspace_bytes(c["P"], c["I"])), dtype=torch.uint8, device="cuda")
        Yp = torch.zeros_like(want)
        sides = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        for _ in range(3):
            for stream, (lo, hi) in zip(sides, ((0, 3), (3, 6))):
                with torch.cuda.stream(stream):
                    moe.moe_expert_group_forward_mx(lo, hi, c["x"], None, 1, c["off"], c["Wg"], c["Wu"], c["Wd"], Yp, ws)
        torch.cuda.synchronize()
        assert torch.equal(bits(Yp), bits(want))


def test_more_tiles_than_a_grid_has_in_its_second_dimension(moe):
    """Short contractions take any number of rows, in tiles of 32."""
    period, E, H, I = 499, 2, 64, 128
    counts = [1_300_000, 1_000_001]
    small = block_case(moe, [period, period], H, I, 12)
    check_block(small, run_block(moe, small))
    want = run_block(moe, small)
    at = torch.cat([torch.arange(n, device="cuda") % period + period * e for e, n in enumerate(counts)])
    c = dict(small, P=sum(counts), counts=counts, x=tuple(t.view(torch.uint8)[at].view(t.dtype) for t in small["x"]),
             off=torch.tensor([0, counts[0], sum(counts)], dtype=torch.int32).cuda())
    assert sum(counts) // 32 > 65535
    assert torch.equal(bits(run_block(moe, c)), bits(want[at]))


def test_rows_beyond_four_gigabytes(moe):
    period, H, T = 1009, 64, (1 << 23) + 77
    x = rows(period, H, 8).cuda()
    y = rows(period, H, 9).cuda()
    at = torch.arange(T, device="cuda") % period
    full = moe.moe_residual_norm_mx(x, y)
    got = moe.moe_residual_norm_mx(x[at], y[at])
    for a, b in zip(got, full):
        assert torch.equal(bits(a), bits(b)[at])
    del got
    H, T = 16384, 140_003                                      # 4.6 GB of bf16, 2.3 GB of bytes
    x = rows(7, H, 10).cuda()
    at = torch.arange(T, device="cuda") % 7
    q, s = moe.moe_quantize_mx(x)
    big = x[at]
    gq, gs = moe.moe_quantize_mx(big)
    for lo in (0, 65_536, T - 5):
        assert torch.equal(gq.view(torch.uint8)[lo:lo + 5], q.view(torch.uint8)[at[lo:lo + 5]])
    assert torch.equal(gs.view(torch.uint8), s.view(torch.uint8)[at])
