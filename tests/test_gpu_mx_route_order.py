"""Gating by scores where the order of additions decides: the ids are the definition's though the products run on matrix cores."""
import pytest
import torch

from tests import mx_reference as ref
from tests.test_gpu_mx import check_route, moe  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def two_rows(H, lanes, scale, shift):
    """A token and two router rows whose logits, near 0, the defined order gets wrong by as much as it can, in opposite directions:
    its first `lanes` partial sums (the rest are zero but for one) take one large product and then only products of half a unit
    in the last place of it, a little less where the rounding is to go down and a little more where it is to go up.  In exact
    arithmetic the first logit is larger by `shift` * 2^-24 of the sum of all magnitudes."""
    x, w = torch.zeros(1, H, dtype=torch.float64), torch.zeros(2, H, dtype=torch.float64)
    for lane in range(lanes):
        sign = 1.0 if lane % 2 == 0 else -1.0
        at = [512 * c + 8 * lane + i for c in range(-(-H // 512)) for i in range(8) if 512 * c + 8 * lane + i < H]
        x[0, at[0]], w[:, at[0]] = scale, sign * scale
        x[0, at[1:]] = scale * 2.0 ** -12
        up, down = sign * scale * 2.0 ** -12 * (1 + 2.0 ** -7), sign * scale * 2.0 ** -12 * (1 - 2.0 ** -8)
        w[0, at[1:]], w[1, at[1:]] = (down, up) if sign > 0 else (up, down)
    x[0, 8 * lanes] = scale * 2.0 ** -8
    w[0, 8 * lanes] = shift * 2.0 ** -24 * lanes * scale * 2.0 ** 8
    return x.to(torch.bfloat16), w.to(torch.bfloat16)


@pytest.mark.parametrize("H,shifts", [(2112, (60, 66, 68, 70, 72, 74)), (2048, (56, 58, 60)), (4160, (120, 130, 134, 138)), (8128, (230, 240))])
@pytest.mark.parametrize("score,balance", [("sigmoid", False), ("sigmoid", True), ("softmax", False), ("softmax", True)])
def test_route_scored_where_the_defined_order_rounds_as_badly_as_it_can(moe, H, shifts, score, balance):
    print(f"[case] worst order H={H} {score} balance={balance}", flush=True)
    for scale in (2.0 ** 5, 2.0 ** 3, 1.0):
        for shift in shifts:
            x, Wr = two_rows(H, 8, scale, float(shift))
            l = ref.logits(x, Wr)[0].double()
            true = (x.double() @ Wr.double().T)[0]
            assert float(l[1]) > float(l[0]) and float(true[0]) > float(true[1])
            for rows in ([0, 1], [1, 0]):
                b = torch.zeros(2) if balance else None
                check_route(moe, x, Wr[rows].contiguous(), b, 1, score, 1, 1, 1, False, 1.0)
                for best in (1, 2):        # the same between groups: each of the two, and 3 experts that nobody wants
                    far = torch.zeros(8, H, dtype=torch.bfloat16)
                    far[:, 0] = -16.0
                    far[0], far[4] = Wr[rows[0]], Wr[rows[1]]
                    if best == 2:
                        far[1], far[5] = Wr[rows[0]], Wr[rows[1]]
                    check_route(moe, x, far, torch.zeros(8) if balance else None, best, score, 2, 1, best, False, 1.0)


def hard_sums(H, T, seed):
    """Tokens whose products with a router row of ones and twos are hard to add: values that cancel, beside many just below what an
    instruction keeps, at random places; a sum of 3 or so is left."""
    g = torch.Generator().manual_seed(seed)
    x = torch.zeros(T, H, dtype=torch.float64)
    big = 2.0 ** 10
    for t in range(T):
        kind = t % 4
        at = torch.randperm(H, generator=g)
        if kind == 3:                                          # anything
            x[t] = torch.randn(H, generator=g).double() * 2.0 ** torch.randint(-16, 9, (H,), generator=g).double()
            x[t] -= x[t].to(torch.bfloat16).double().sum() / H
        else:                                                  # one pair of large values and small ones of one sign or both
            x[t] = big * 2.0 ** -24 * (0.5 + 0.49 * torch.rand(H, generator=g).double() * (1 + (t // 4) % 5))
            if kind == 1:
                x[t] *= torch.randint(0, 2, (H,), generator=g).double() * 2 - 1
            first, last = (at[0], at[1]) if kind < 2 else (0, H - 1)
            x[t, first], x[t, last] = big, -big
        x[t, at[2]] = 3.0
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("H", [64, 512, 2048, 2112])
def test_logits_of_the_matrix_cores_are_within_the_bound_that_the_choice_counts_on(moe, H):
    """Two experts, one with a router row of zeros: the weights tell the other one's logit as the matrix cores add it (it is far
    enough from 0 that it need not be formed again).  An instruction's group of 8: 8 units of 2^-24 of its largest product; then
    one of all that is summed so far; 7 for the parts."""
    print(f"[case] matrix core logits H={H}", flush=True)
    T = 256
    x = hard_sums(H, T, H)
    Wr = torch.zeros(2, H, dtype=torch.bfloat16)
    Wr[0] = 1.0
    ids, w = moe.moe_route_scored(x.cuda(), Wr.cuda(), None, 2, "softmax")
    w, ids = w.cpu().double(), ids.cpu()
    got = torch.where(ids[:, 0] == 0, 1.0, -1.0) * (w[:, 0].log() - w[:, 1].log())
    p, u, steps = x.double(), 2.0 ** -24, H // 64
    bound = torch.zeros(T, dtype=torch.float64)
    for part in range(8):
        groups = p[:, 64 * (steps * part // 8):64 * (steps * (part + 1) // 8)].abs().reshape(T, -1, 8)
        if groups.shape[1]:
            bound += 8 * groups.amax(-1).sum(1) + groups.sum(-1).cumsum(1).sum(1) + 7 * groups.sum((1, 2))
    exact = p.sum(1)
    spread = 2 * 1.1 * (29 + 16 * -(-steps // 8)) * u * p.norm(dim=1) * H ** 0.5           # (closer than that it may be formed again)
    sure = (exact.abs() > spread) & (exact.abs() < 12.0)
    assert int(sure.sum()) > T // 2
    # a weight in fp32: the rounded difference of logits below 12 (2^-21), the exponential (2 units: 2^-22), sum, quotient and the
    # weight itself (2^-24 each); two of them make the logit: less than 2^-19
    d = (got - exact).abs()
    assert bool((d <= 1.01 * u * bound + 2.0 ** -19)[sure].all()), float((d / (u * bound))[sure].max())
    print(f"largest error {float((d / (u * bound))[sure].max()):.3f} of the bound", flush=True)


@pytest.mark.parametrize("T,H,E,K,score,groups,top,best,renorm,balance", [
    (37, 512, 60, 4, "softmax", 1, 1, 1, False, False), (300, 2048, 256, 8, "sigmoid", 8, 4, 2, True, True),
    (5000, 320, 256, 16, "softmax", 8, 3, 1, True, True), (64, 1088, 160, 6, "softmax", 4, 2, 2, False, True), (9, 64, 16, 16, "sigmoid", 1, 1, 1, False, False)])
def test_weights_of_logits_that_any_order_adds_exactly(moe, T, H, E, K, score, groups, top, best, renorm, balance):
    """Whole numbers times sixteenths: every partial sum is a float, so nothing is left but the scores.  In units of 2^-24: an
    exponential 4 (two in the last place), the denominator 4 + 21 additions in a row, quotient and scale 1 each; with renorm the
    denominator is common, and the chosen scores' sum is 5 + 15 additions: below 32 in all."""
    print(f"[case] exact logits {T} {H} {E} {K} {score} {groups}", flush=True)
    g = torch.Generator().manual_seed(T + H)
    x = torch.randint(-2, 3, (T, H), generator=g).to(torch.bfloat16)
    Wr = (torch.randint(-3, 4, (E, H), generator=g) * (torch.rand((E, H), generator=g) < 64.0 / H) / 16.0).to(torch.bfloat16)
    b = torch.randint(-8, 9, (E,), generator=g) / (256.0 if score == "sigmoid" else 256.0 * E) if balance else None
    ids, w = check_route(moe, x, Wr, b, K, score, groups, top, best, renorm, 2.5)
    rid, rw = ref.route(x, Wr, b, K, score, groups, top, best, renorm, 2.5)
    assert torch.equal(ids.cpu(), rid)
    assert bool(((w - rw).abs() <= 2.0 ** -19 * rw.abs() + 1e-37).all()), float(((w - rw).abs() / rw.abs().clamp_min(1e-30)).max())
