"""The margins of moe_route_scored's choice (csrc/score_margin.h) on the CPU: what a logit may be off by moves no compared value, and
no difference of two groups' values, by more than its margin; and the count of roundings behind that bound."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_26881_amd", "csrc")
SOURCE = """
#include "score_margin.h"
static moe::ScoreMargin of(int form, float doubt, float largest, float bal) {
  return form == 0 ? moe::margin_of_sigmoids(doubt) : form == 1 ? moe::margin_of_logits(doubt) : moe::margin_of_softmax(doubt, largest, bal);
}
extern "C" {
float off(int form, float doubt, float largest, float bal, float c) { return of(form, doubt, largest, bal).off(c); }
float between(int form, float doubt, float largest, float bal, int best, float size) { return of(form, doubt, largest, bal).between_groups(best, size); }
int roundings(int k, int k_end, int steps) { return moe::logit_roundings(k, k_end, steps); }
float most() { return moe::LOGIT_ERROR_MOST; }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("margin")
    (d / "m.cc").write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(d / "m.cc"), "-o", str(d / "m.so")], check=True)
    so = ctypes.CDLL(str(d / "m.so"))
    f = ctypes.c_float
    so.off.restype = so.between.restype = so.most.restype = f
    so.off.argtypes = [ctypes.c_int, f, f, f, f]
    so.between.argtypes = [ctypes.c_int, f, f, f, ctypes.c_int, f]
    return so


SIGMOID, LOGIT, SOFTMAX = 0, 1, 2


def compared(form, l, b):
    s = torch.sigmoid(l) if form == SIGMOID else l if form == LOGIT else torch.softmax(l, -1)
    return s, s + b


CASES = [(f, d, s, b) for f in (SIGMOID, LOGIT, SOFTMAX) for d in (1e-6, 1e-3, 1.0 / 32.0)
         for s, b in ((0.01, 0.0), (1.0, 0.0), (1.0, 0.3), (4.0, 0.05), (4.0, 3.0), (0.1, 0.001)) if f != LOGIT or b == 0.0]


@pytest.mark.parametrize("form,doubt,spread,bal", CASES)
def test_margins_cover_what_logits_are_off_by(lib, form, doubt, spread, bal):
    """Errors of +-doubt on the logits, those that move the difference of two groups' values by the most among them.  The bounds are
    compared with 64-bit values: their allowance for fp32 is on top."""
    assert doubt <= lib.most()
    g = torch.Generator().manual_seed(int(1e6 * doubt) + 7)
    for trial in range(20):
        l = torch.randn(16, generator=g, dtype=torch.float64) * spread
        b = torch.randn(16, generator=g, dtype=torch.float64) * bal
        s, c = compared(form, l, b)
        for best in (1, 2):
            if bal or trial % 2:              # the best (two) of groups 0 and 1 change places in value: alike, though their scores differ
                for j in range(best):
                    d = (c[j] - c[4 + j]) / 2
                    shift = (c[:8].max() - c[:8].min()) * (0.1 if bal else 0.0)
                    if bal:
                        b[j], b[4 + j] = b[j] - d + shift, b[4 + j] + d + shift
                    elif form == LOGIT or form == SIGMOID:
                        l[4 + j] = l[j]
                s, c = compared(form, l, b)
            largest, most = float(s.max()), float(b.abs().max())
            top = c.reshape(4, 4).topk(best, dim=1)
            at = top.indices + 4 * torch.arange(4)[:, None]
            value, size = top.values.sum(1), top.values.abs().sum(1)
            moved = [lib.between(form, doubt, largest, most, best, float(v)) for v in size]
            own = torch.tensor([lib.off(form, doubt, largest, most, abs(float(v))) for v in c], dtype=torch.float64)
            for p, q in ((0, 1), (1, 0), (2, 0), (3, 1)):
                for others in (-1.0, 1.0, 0.0):                # p's experts up, q's down, the others either way (the denominator)
                    e = torch.full((16,), others, dtype=torch.float64)
                    e[at[p]], e[at[q]] = 1.0, -1.0
                    c1 = compared(form, l + doubt * e, b)[1]
                    assert bool(((c1 - c).abs() <= own).all()), (best, p, q)
                    if abs(float(value[p] - value[q])) <= 1e-9 * float(size.max()):      # (values that are alike)
                        change = abs(float(c1[at[p]].sum() - c1[at[q]].sum()))
                        assert change <= max(moved[p], moved[q]), (best, p, q, change, moved[p], moved[q])


@pytest.mark.parametrize("H", [64, 192, 512, 576, 2048, 2112, 4160, 8128, 8192])
def test_roundings_are_at_least_those_on_the_way(lib, H):
    steps = H // 64
    for part in range(8):
        k0, k1 = steps * part // 8, steps * (part + 1) // 8
        for k in range(k0, k1):
            # products: the cuts of a group whose largest term this is, the groups from its own to the end of the part, the parts
            mine = 8 + (k1 - k) * 64 // 8 + 7
            # the defined order, from the step's first element on: the later elements of its lane, itself, six folds
            lane = (64 * k // 8) % 64
            later = sum(1 for h in range(H) if (h // 8) % 64 == lane and h >= 64 * k)
            assert lib.roundings(k, k1, steps) >= mine + later + 6
