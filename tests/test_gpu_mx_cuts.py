"""The 8-bit expert blocks give the same bits however the experts are cut into blocks, where the cut changes which form of the
streaming kernel runs: the whole layer's down projection has more blocks of columns than the card has compute units, a cut fewer."""
import pytest
import torch

from tests.test_gpu_mx import bits, block_case, check_block, moe, run_block  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def cancelling(moe, counts, H, I, seed):
    """Hidden values in equal pairs with opposite weights but for one in 32: the sums are far smaller than their terms, so another
    order of additions shows in almost every output."""
    c = block_case(moe, counts, H, I, seed)
    half = I // 2
    for w in ("Wg", "Wu"):
        for t in c[w]:
            t.view(torch.uint8)[:, half:] = t.view(torch.uint8)[:, :half]
    q, s = (t.view(torch.uint8) for t in c["Wd"])
    s[..., half // 32:] = s[..., :half // 32]
    q[..., half:] = q[..., :half] ^ 0x80
    q[..., half::32] ^= 0x01                                   # one step of e4m3
    return c


@pytest.mark.parametrize("counts,H,I", [([1, 2] * 30, 2048, 1408), ([1, 0, 2, 1, 5, 0] * 10, 2048, 2048), ([1] * 48, 1024, 2880), ([12, 3, 9] * 8, 1408, 768)],
                         ids=["60x2048x1408", "60x2048x2048", "48x1024x2880", "24x1408x768"])
def test_rows_do_not_depend_on_the_block_cut_across_the_forms_of_the_streaming_kernel(moe, counts, H, I):
    print(f"[case] cuts experts={len(counts)} H={H} I={I}", flush=True)
    E = len(counts)
    assert min(E, sum(counts)) * (H // 64) > 256 >= 4 * (H // 64)
    for c in (block_case(moe, counts, H, I, H + I), cancelling(moe, counts, H, I, H + I + 1)):
        whole = run_block(moe, c)
        for n in (1, 4, 15):
            cut = run_block(moe, c, [(lo, min(lo + n, E)) for lo in range(0, E, n)])
            off = bits(cut) != bits(whole)
            assert not bool(off.any()), f"blocks of {n}: {int(off.sum())} of {off.numel()} outputs differ"
    check_block(block_case(moe, counts, H, I, H + I), run_block(moe, block_case(moe, counts, H, I, H + I)))


def test_two_blocks_at_once_of_another_form_than_the_whole_layer(moe):
    c = cancelling(moe, [2, 1] * 30, 2048, 1408, 5)
    want = run_block(moe, c)
    ws = torch.empty(int(moe.load().moe_expert_workspace_bytes(c["P"], c["I"])), dtype=torch.uint8, device="cuda")
    Yp = torch.zeros_like(want)
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for at in range(0, 60, 4):
        with torch.cuda.stream(sides[at // 4 % 2]):
            moe.moe_expert_group_forward_mx(at, at + 4, c["x"], None, 1, c["off"], c["Wg"], c["Wu"], c["Wd"], Yp, ws)
    torch.cuda.synchronize()
    assert torch.equal(bits(Yp), bits(want))
