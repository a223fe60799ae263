"""NaN blocks of weights that are in use reach the outputs that they enter, and no others."""
import pytest
import torch

from tests.test_gpu_mx import bits, block_case, moe, run_block  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu

# two experts in use and one that is not; a few rows, tiles of 16 and 32, and the tile kernel, with whole and half steps
SIZES = [([3, 0, 2], 256, 192), ([1, 0, 1], 2048, 1408), ([40, 0, 33], 256, 192), ([20, 0, 15], 448, 576), ([200, 0, 90], 512, 576), ([70, 0, 300], 1088, 704)]


@pytest.mark.parametrize("counts,H,I", SIZES, ids=lambda v: str(v).replace(" ", "") if isinstance(v, list) else str(v))
@pytest.mark.parametrize("how", ["block", "scale", "value"])
def test_nan_of_a_weight_reaches_the_outputs_that_it_enters(moe, counts, H, I, how):
    print(f"[case] NaN weights counts={counts} H={H} I={I} {how}", flush=True)
    rows0 = counts[0]

    def spoilt(name, row, block):
        c = block_case(moe, counts, H, I, H + I)
        q, s = (t.view(torch.uint8) for t in c[name])
        if how in ("block", "scale"):
            s[0, row, block] = 255
        if how == "block":
            q[0, row, 32 * block:32 * block + 32] = 0x7F
        if how == "value":
            q[0, row, 32 * block + 5] = 0x7F
        return c

    want = run_block(moe, block_case(moe, counts, H, I, H + I))
    # a row of the down projection: one column of that expert's outputs
    for row, block in ((0, 0), (H - 1, I // 32 - 1), (37, 3)):
        got = run_block(moe, spoilt("Wd", row, block))
        assert bool(torch.isnan(got[:rows0, row]).all()), (row, block)
        keep = torch.ones(got.shape, dtype=torch.bool, device=got.device)
        keep[:rows0, row] = False
        assert torch.equal(bits(got)[keep], bits(want)[keep])
    # a row of the gate or up projection: one hidden value, which every output of that expert's rows takes
    for name in ("Wg", "Wu"):
        for row, block in ((0, 0), (I - 1, H // 32 - 1), (33, 2)):
            got = run_block(moe, spoilt(name, row, block))
            assert bool(torch.isnan(got[:rows0]).all()), (name, row, block)
            assert torch.equal(bits(got[rows0:]), bits(want[rows0:]))
