"""The weight that a cached key has drawn does not depend, to the last bit, on how a call is launched: one launch or several, alone or in a
batch, whatever max_len bounds the lengths."""
import numpy as np
import pytest

import cache_plain as plain
from test_cache_ops_gpu import Case, dev, ia, torch, wide  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d, page", [(64, 16), (128, 64), (64, 24)])
@pytest.mark.parametrize("G, L", [(1, 1), (4, 4), (17, 1), (5, 8), (3, 23), (16, 14)])  # 1, 16, 17, 40, 69 and 224 rows
def test_weights_do_not_depend_on_the_launches(torch, ia, d, page, G, L):
    from paper_2511_21513_amd import binding

    most, lens = 18000 // page * page, [1500, 700, 2, 1321]  # a table for so many keys leads to the launches of long sequences
    c = Case(torch, G + L, 4, 2, d, page, lens, room=0)
    rng = np.random.default_rng(G * L)
    q, s, qt, st = c.queries(torch, 2 * G, L)
    w = rng.random((4, 2, c.width * page)).astype(np.float32)
    wt = dev(torch, w)
    want_out, _, _, want = plain.attend(q, s, c.k, c.v, c.table, c.lens, c.sk, c.sv, weight=w, decay=np.float32(0.75))

    def run(table, rows, planes, **more):
        cache = binding.PagedCache(c.t["k"], c.t["v"], table[rows].contiguous(), c.t["lens"][rows].contiguous(), c.t["sk"], c.t["sv"])
        out = torch.full_like(planes[rows], -1)
        got = ia.cache_forward(cache, qt[rows].contiguous(), st[rows].contiguous(), dtype=torch.int8, weight=planes[rows], weight_out=out, decay=0.75, **more)
        return got, out[:, :, :c.width * page]

    every, table = slice(0, 4), c.t["table"]
    long = torch.full((4, most // page), -1, dtype=torch.int32, device="cuda")
    long[:, :c.width] = table
    planes = torch.zeros((4, 2, most), device="cuda")
    planes[:, :, :c.width * page] = wt
    many = torch.arange(4, device="cuda").repeat(60)  # in a batch that fills the chip
    got, out = run(table, every, wt)
    others = [run(long, every, planes), run(long, every, planes, max_len=c.width * page), run(long, every, planes, max_len=9000)] + [run(table, slice(b, b + 1), wt) for b in range(4)]
    others += [run(table, many, wt), run(long, many, planes)]
    torch.cuda.synchronize()
    under = torch.arange(out.shape[2], device="cuda")[None, None] < c.t["lens"][:, None, None]
    assert (np.abs(wide(out) - want) <= (G * L + 3) * 2.0 ** -24 * want)[under.expand(out.shape).cpu().numpy()].all()
    for i, (g, o) in enumerate(others):
        rows = [0, 1, 2, 3] if i < 3 else [i - 3] if i < 7 else many.tolist()
        assert torch.equal(g, got[rows]), i
        assert torch.equal(torch.where(under[rows], o, 0.0), torch.where(under[rows], out[rows], 0.0)), i
