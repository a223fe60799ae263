"""Softmax scores that round to the same fp32 though their logits differ: the lower id wins, also where other experts, with logits equal
to the last choice's, stand between the two."""
import pytest
import torch

from tests import mx_reference as ref
from tests.test_gpu_mx import check_route, moe  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def alike(E, low, high, T, H, seed):
    """Tokens for which the experts `low` have logit 1/4, the experts `high` a unit in the last place more, and the others far less,
    by another amount for every token (which moves the denominator, and with it where scores round)."""
    g = torch.Generator().manual_seed(seed)
    x, Wr = torch.zeros(T, H), torch.zeros(E, H)
    at = torch.randperm(H - 3, generator=g)[:3] + 3
    x[:, at[0]], x[:, at[1]] = 1.0, 2.0 ** -17
    x[:, at[2]] = 1.0 + torch.rand(T, generator=g) * 2
    Wr[:, at[2]] = -1.0
    for e in low + high:
        Wr[e, at[0]], Wr[e, at[2]] = 0.25, 0.0
        Wr[e, at[1]] = 2.0 ** -8 if e in high else 0.0
    return x.to(torch.bfloat16), Wr.to(torch.bfloat16)


CASES = [  # E, experts of the lower logit, of the higher one, K, groups, top_groups
    (5, [0], [1, 2, 3], 2, 1, 1), (5, [0], [1, 2], 1, 1, 1), (8, [2, 0], [3, 5, 6, 7], 3, 1, 1), (60, [11], [20, 31, 40], 2, 1, 1),
    (256, [3, 70], [100, 200, 201, 255], 2, 1, 1), (8, [0], [2, 4, 6], 1, 4, 1), (8, [1], [2, 4, 6], 2, 4, 2), (96, [5], [17, 40, 80], 2, 12, 2),
    (256, [0], [60, 130, 200], 1, 8, 1), (16, [0, 5], [9, 10, 15], 2, 16, 2), (5, [4], [1, 2, 3], 2, 1, 1), (8, [6], [2, 3, 5], 2, 8, 2),
]


@pytest.mark.parametrize("E,low,high,K,groups,top", CASES, ids=lambda v: str(v).replace(" ", "") if isinstance(v, list) else str(v))
def test_scores_that_round_alike_behind_equal_logits(moe, E, low, high, K, groups, top):
    print(f"[case] alike E={E} low={low} high={high} K={K} groups={groups}", flush=True)
    met = 0
    for H, seed in ((64, 1), (2048, 2), (576, 3)):
        x, Wr = alike(E, low, high, 96, H, seed)
        ids, _ = check_route(moe, x, Wr, None, K, "softmax", groups, top, 1, True, 1.0)
        check_route(moe, x, Wr, None, K, "softmax", groups, top, 1, False, 2.5)
        met += int(torch.isin(ids.cpu(), torch.tensor(low, dtype=torch.int32)).any(1).sum())
    if min(low) < min(high):
        assert met > 0      # (scores did round alike)
