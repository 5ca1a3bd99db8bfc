"""INT8 output of attention over the paged cache at every ratio s_V / (255 s_O): past what a multiplier of 31 bits and a shift can stand for
it is the formula's value all the same, +-127 or 0, and the keys' weights are those of any other output."""
import math
from fractions import Fraction

import numpy as np
import pytest

import cache_plain as plain
from test_cache_ops_gpu import Case, dev, ia, torch, wide  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

# 1.9 2^29 and 2^30 (1 - 2^-33), which rounds to 2^30: both sides of the multiplier's range; 2^-32, half of it; the largest and the smallest there are
RATIOS = [0.3, 1.9 * 2.0 ** 29, 2.0 ** 30, 2.0 ** 31, 1e20, 1e35, 2.0 ** -31, 2.0 ** -32, 2.0 ** -33, 1e-35, 5e-41]


def formula(acc, sv, so):
    r = Fraction(float(sv)) / (255 * Fraction(float(so)))
    return np.array([min(max(math.floor(int(a) * r + Fraction(1, 2)), -127), 127) for a in acc.ravel()]).reshape(acc.shape)


@pytest.mark.parametrize("lens", [[1, 40, 130], [9000, 65, 0]], ids=str)  # in one launch, and with the keys split
@pytest.mark.parametrize("L", [1, 3, 9])  # 2, 6 and 18 rows: with several blocks of rows
def test_output_scales_of_all_sizes(torch, ia, lens, L):
    Hkv = len(RATIOS)
    c = Case(torch, 7 + L, len(lens), Hkv, 64, 16, lens, room=0)
    c.v[:, 0] = 0  # accumulators of 0: 0 at any ratio
    c.sv[:] = np.float32(0.01)
    c.up(torch)
    q, s, qt, st = c.queries(torch, 2 * Hkv, L)
    so = np.repeat(c.sv.astype(np.float64) / 255 / np.array(RATIOS), 2)
    so[0] = 1e-40
    so = np.maximum(so, 1e-45).astype(np.float32)  # the greatest ratio there is: of the smallest subnormal number
    assert (so > 0).all() and np.isfinite(so).all()
    w = c.rng.random((c.B, Hkv, c.width * c.page)).astype(np.float32)
    got_w, other_w = dev(torch, w), dev(torch, w)
    got = ia.cache_forward(c.cache, qt, st, dtype=torch.int8, scale_out=dev(torch, so), weight=got_w, decay=0.5)
    ia.cache_forward(c.cache, qt, st, dtype=torch.float32, weight=other_w, decay=0.5)
    torch.cuda.synchronize()
    acc, _, _, new = plain.attend(q, s, c.k, c.v, c.table, c.lens, c.sk, c.sv, weight=w, decay=0.5)
    assert (np.abs(acc[0]) > 0).any()
    for head in range(2 * Hkv):
        sv = c.sv[head // 2]
        r = float(sv) / (255.0 * float(so[head]))
        inside = 1 <= 31 - math.frexp(r)[1] <= 62
        want = plain.requantize(acc[:, head], sv, so[head]) if inside else formula(acc[:, head], sv, so[head])
        assert (got[:, head].cpu().numpy() == want).all(), r
        if r > 1e9:
            assert (want == 127 * np.sign(acc[:, head])).all()
    assert torch.equal(got_w, other_w)
    assert (np.abs(wide(got_w) - new) <= (2 * L + 3) * 2.0 ** -24 * new).all()
