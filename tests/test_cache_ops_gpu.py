"""GPU tests of the operators around the paged cache against plain forms in 64 bits (cache_plain.py).  Integers have to be equal; a
floating-point result may be off by half a step of its type (torch.finfo(t).eps / 2 of the value) for each rounding on its way."""
import math

import numpy as np
import pytest

import cache_plain as plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch

    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X (torch.cuda.is_available() is False)")
    return torch


@pytest.fixture(scope="module")
def ia(torch):
    from paper_2511_21513_amd import binding

    c = binding.IntAttn(device=0)
    yield c
    torch.cuda.synchronize()
    c.close()


def dev(torch, x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(getattr(torch, dtype))


def wide(t):
    return t.double().cpu().numpy()


def half_step(torch, dtype):
    return torch.finfo(getattr(torch, dtype)).eps / 2


# ---------------------------------------------------------------- rope

ROPES = [
    # dtype, B, L, heads, d, rot, axes, halves, far, inverse
    ("float32", 1, 1, (1,), 16, 16, 1, False, 1, False),
    ("float32", 2, 5, (3, 1), 64, 64, 1, False, 100000, False),
    ("float32", 1, 9, (2, 2), 128, 32, 3, True, 5000, True),
    ("bfloat16", 3, 1, (8, 2), 128, 128, 1, False, 1000000, False),
    ("bfloat16", 2, 33, (5,), 80, 48, 2, True, 4096, False),
    ("float16", 1, 130, (4, 4), 64, 64, 3, True, 2000, True),
    ("float16", 2, 7, (1, 1), 256, 256, 4, False, 70000, False),
    ("float16", 1, 3, (2,), 1024, 256, 2, False, 70000, True),
    ("bfloat16", 1, 300, (33, 7), 64, 16, 2, True, 30, False),
    ("float32", 3, 700, (1, 1), 64, 32, 1, False, 4000, False),      # many tokens to a workgroup
    ("float16", 7, 401, (1,), 16, 16, 1, True, 4000, True),
    ("bfloat16", 1, 5, (257, 1), 1024, 256, 4, False, 300, False),
]


def rope_case(seed, B, L, heads, d, rot, axes, far):
    rng = np.random.default_rng(seed)
    xs = [rng.standard_normal((B, h, L, d)).astype(np.float32) * 2 for h in heads]
    pos = rng.integers(-far, far + 1, (axes, B, L)).astype(np.int32)
    freq = 10000.0 ** (-2.0 * np.arange(rot // 2) / rot)
    axis = [int(a) for a in rng.integers(0, axes, rot // 2)]
    return xs, pos, freq, axis


@pytest.mark.parametrize("layout", ["heads first", "tokens first", "in place"])
@pytest.mark.parametrize("case", ROPES, ids=str)
def test_rope(torch, ia, case, layout):
    dtype, B, L, heads, d, rot, axes, halves, far, inverse = case
    xs, pos, freq, axis = rope_case(len(str(case)), B, L, heads, d, rot, axes, far)
    ts = [dev(torch, x, dtype) for x in xs]
    if layout == "tokens first":
        ts = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in ts]
    want = [plain.turned(wide(t), pos, freq, axis, halves, inverse) for t in ts]
    before = [t.clone() for t in ts]
    got = ia.rope(ts, dev(torch, pos), dev(torch, freq), axis=axis, pairing="halves" if halves else "adjacent", inverse=inverse, out=ts if layout == "in place" else None)
    torch.cuda.synchronize()
    for t, b, g, w in zip(ts, before, got, want):
        if layout != "in place":
            assert torch.equal(t, b)
        # roundings: to 32 bits, and to the type; the angle's product in 64 bits, by 2^-53 of up to far radians, turns by as much
        size = np.abs(wide(b)).max()
        limit = (half_step(torch, dtype) * 1.0001 + (2.0 ** -24 if dtype != "float32" else 0)) * np.abs(w) + size * (far * 2.0 ** -51 + 2.0 ** -50) + (2.0 ** -25 if dtype == "float16" else 0)
        assert (np.abs(wide(g) - w) <= limit).all()
        assert torch.equal(g[..., rot:], b[..., rot:])


def test_rope_is_undone_by_its_inverse_and_is_its_own_gradient(torch, ia):
    xs, pos, freq, axis = rope_case(3, 2, 19, (3,), 64, 64, 3, 9000)
    x, p, f = dev(torch, xs[0]), dev(torch, pos), dev(torch, freq)
    turn = lambda t, inverse: ia.rope(t, p, f, axis=axis, inverse=inverse)
    back = turn(turn(x, False), True)
    assert (back - x).abs().max().item() <= 4 * 2.0 ** -24 * x.abs().max().item() * 2 ** 0.5
    # the gradient of sum(g * rope(x)) by x is rope's inverse on g: against differences of the plain form in 64 bits
    rng = np.random.default_rng(5)
    g = rng.standard_normal(x.shape).astype(np.float32)
    grad = wide(turn(dev(torch, g), True))
    for _ in range(20):
        at = tuple(int(rng.integers(0, n)) for n in x.shape)
        step = np.zeros(x.shape)
        step[at] = 0.5
        slope = ((plain.turned(xs[0] + step, pos, freq, axis, False) - plain.turned(xs[0] - step, pos, freq, axis, False)) * g).sum()
        assert abs(grad[at] - slope) <= 2.0 ** -24 * abs(slope) + 1e-10 * 9000
    # torch's own gradient through a rotation written out
    y = x.clone().requires_grad_(True)
    ang = (p[torch.tensor(axis, device="cuda")].permute(1, 2, 0).double() * f)[:, None]
    a, b = y[..., 0::2].double(), y[..., 1::2].double()
    z = torch.stack((a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos()), dim=-1).flatten(-2)
    z.backward(dev(torch, g).double())
    assert (turn(dev(torch, g), True).double() - y.grad.double()).abs().max().item() <= 2.0 ** -23 * float(np.abs(g).max()) * 2


# ---------------------------------------------------------------- a cache

class Case:
    """A pool of pages filled with integers, tables without order, lengths as given; numpy arrays and their tensors."""

    def __init__(self, torch, seed, B, Hkv, d, page, lens, per_head=True, spare=3, room=1):
        from paper_2511_21513_amd import binding

        rng = self.rng = np.random.default_rng(seed)
        width = max(1, max(-(-max(n, 0) // page) for n in lens) + room)
        self.n_pages = B * width + spare
        self.k = rng.integers(-127, 128, (self.n_pages, Hkv, page, d)).astype(np.int8)
        self.v = rng.integers(-128, 128, (self.n_pages, Hkv, page, d)).astype(np.int8)
        self.table = rng.permutation(self.n_pages)[:B * width].reshape(B, width).astype(np.int32)
        self.lens = np.array(lens, dtype=np.int32)
        n = Hkv if per_head else 1
        self.sk, self.sv = (rng.uniform(0.005, 0.03, n).astype(np.float32) for _ in range(2))
        self.B, self.Hkv, self.d, self.page, self.width, self.per_head = B, Hkv, d, page, width, per_head
        self.up(torch)

    def up(self, torch):
        from paper_2511_21513_amd import binding

        self.t = {x: dev(torch, getattr(self, x)) for x in ("k", "v", "table", "lens", "sk", "sv")}
        self.cache = binding.PagedCache(*(self.t[x] for x in ("k", "v", "table", "lens", "sk", "sv")))

    def queries(self, torch, Hq, L, size=1.0):
        q = self.rng.integers(-127, 128, (self.B, Hq, L, self.d)).astype(np.int8)
        s = (self.rng.uniform(0.002, 0.02, (self.B, Hq, L)) * size).astype(np.float32)
        return q, s, dev(torch, q), dev(torch, s)


FORWARDS = [
    # B, Hq, Hkv, d, page, L, lens, n_new (None: all), per_head
    (1, 1, 1, 64, 16, 1, [1], None, False),
    (1, 4, 1, 128, 64, 1, [64], None, True),
    (3, 8, 2, 128, 16, 1, [0, 63, 65], None, True),
    (2, 8, 8, 64, 16, 1, [200, 17], None, False),
    (2, 6, 2, 128, 24, 1, [191, 48], None, True),      # pages that end inside a step
    (2, 4, 4, 64, 1, 1, [70, 3], None, True),          # a page for each key
    (2, 8, 2, 64, 8, 3, [129, 2], None, True),         # rows before the first key
    (4, 8, 2, 128, 32, 4, [300, 4, 77, 9], [4, 2, 0, 9], True),
    (1, 32, 1, 128, 64, 1, [333], None, True),         # two blocks of rows
    (1, 35, 5, 64, 100, 5, [260], [3], False),         # 35 rows a head, seven heads of one
    (2, 3, 3, 128, 16, 1, [1500, 700], None, True),
    (1, 16, 2, 64, 7, 2, [555], None, True),
    (5, 4, 2, 128, 64, 1, [2100, 0, 1, 1025, 64], None, True),   # long, none, one and a step in a batch
    (2, 20, 1, 64, 16, 2, [1300, 3], [2, 1], False),
    (3, 3, 3, 64, 24, 4, [1500, 2, 600], [4, 0, 3], True),
]


def run_forward(torch, ia, c, Hq, L, n_new, dtype="int8", weight=True, size=1.0, scale_out=True, max_len=0, decay=0.75):
    q, s, qt, st = c.queries(torch, Hq, L, size)
    so = c.rng.uniform(0.004, 0.02, Hq if c.per_head else 1).astype(np.float32) if scale_out else None
    slots = c.width * c.page
    w = (c.rng.random((c.B, c.Hkv, slots)) * 2).astype(np.float32) if weight else None
    wt = dev(torch, w) if weight else None
    nn = None if n_new is None else np.array(n_new, dtype=np.int32)
    got = ia.cache_forward(c.cache, qt, st, dtype=getattr(torch, dtype), scale_out=dev(torch, so) if scale_out and dtype == "int8" else None,
                           n_new=None if nn is None else dev(torch, nn), weight=wt, decay=decay, max_len=max_len)
    torch.cuda.synchronize()
    want = plain.attend(q, s, c.k, c.v, c.table, c.lens, c.sk, c.sv, so, nn, w, np.float32(decay), capacity=max_len or None)
    return got, wt, want, w


def check_forward(torch, c, got, wt, want, w, rows, dtype):
    acc, out8, real, new = want
    if dtype == "int8":
        assert int((got.cpu().numpy() != out8).sum()) == 0
    else:  # s_V / 255 to 32 bits, the product, and (16-bit types) the result
        limit = (2 * 2.0 ** -24 + (half_step(torch, dtype) if dtype != "float32" else 0)) * 1.0001 * np.abs(real) + (2.0 ** -25 if dtype == "float16" else 0)
        assert (np.abs(wide(got) - real) <= limit).all()
    if wt is not None:  # each row's quotient, their sum, and the decayed weight's product and sum, all positive
        assert (np.abs(wide(wt) - new) <= (rows + 3) * 2.0 ** -24 * new).all()
        behind = np.arange(w.shape[2])[None, None] >= np.maximum(c.lens, 0)[:, None, None]
        assert (np.where(behind, wide(wt), 0) == np.where(behind, w, 0)).all()


@pytest.mark.parametrize("dtype", ["int8", "bfloat16"])
@pytest.mark.parametrize("case", FORWARDS, ids=str)
def test_forward(torch, ia, case, dtype):
    B, Hq, Hkv, d, page, L, lens, n_new, per_head = case
    c = Case(torch, len(str(case)), B, Hkv, d, page, lens, per_head)
    got, wt, want, w = run_forward(torch, ia, c, Hq, L, n_new, dtype)
    check_forward(torch, c, got, wt, want, w, Hq // Hkv * L, dtype)


@pytest.mark.parametrize("dtype", ["float32", "float16"])
def test_forward_other_types_and_no_weights(torch, ia, dtype):
    c = Case(torch, 4, 2, 2, 64, 16, [130, 31])
    got, wt, want, w = run_forward(torch, ia, c, 8, 1, None, dtype, weight=False)
    check_forward(torch, c, got, wt, want, w, 4, dtype)


@pytest.mark.parametrize("size", [1e-6, 0.02, 50.0, 1e4])
def test_forward_at_all_clip_thresholds(torch, ia, size):
    """Thresholds at the cap of 2^30, past 2^16 and 2^22, of a few units, and of one (rows that one key takes whole: P of 255)."""
    c = Case(torch, 9, 2, 2, 128, 16, [150, 400])
    got, wt, want, w = run_forward(torch, ia, c, 6, 2, None, "int8", size=size, scale_out=False)
    check_forward(torch, c, got, wt, want, w, 6, "int8")


def test_forward_with_pages_that_are_not_there(torch, ia):
    """Hidden keys in front, in between and at the end; a sequence without any; entries on both sides of the pool."""
    c = Case(torch, 21, 4, 2, 64, 16, [100, 90, 40, 200])
    c.table[0, 0], c.table[0, 3] = -1, c.n_pages
    c.table[1, -1], c.table[1, 5] = 2 ** 31 - 1, -2 ** 31
    c.table[2, :] = -7
    c.table[3, 4:9] = 10 ** 6
    c.up(torch)
    for L in (1, 3):
        got, wt, want, w = run_forward(torch, ia, c, 4, L, None)
        check_forward(torch, c, got, wt, want, w, 2 * L, "int8")
        assert int(got[2].abs().sum()) == 0
    # a page for every eight keys, so that a step holds eight of them
    c = Case(torch, 22, 2, 2, 128, 8, [100, 131])
    c.table[:, ::3] = -1
    c.up(torch)
    got, wt, want, w = run_forward(torch, ia, c, 4, 2, None)
    check_forward(torch, c, got, wt, want, w, 4, "int8")


def test_forward_lengths_are_kept_inside_the_table(torch, ia):
    c = Case(torch, 31, 4, 1, 64, 16, [40, 40, 40, 40], room=0)
    c.lens = np.array([-5, 48, 49, 2 ** 31 - 1], dtype=np.int32)  # three pages of 16
    c.up(torch)
    got, wt, want, w = run_forward(torch, ia, c, 2, 1, None)
    assert int((got.cpu().numpy() != want[1]).sum()) == 0
    got, wt, want, w = run_forward(torch, ia, c, 2, 2, [1, -3, 5, 2], max_len=37)
    assert int((got.cpu().numpy() != want[1]).sum()) == 0
    c = Case(torch, 32, 3, 1, 64, 16, [1200, 1200, 1200], room=0)
    c.lens = np.array([-5, 1201, 2 ** 31 - 1], dtype=np.int32)
    c.up(torch)
    got, wt, want, w = run_forward(torch, ia, c, 2, 1, None)
    assert int((got.cpu().numpy() != want[1]).sum()) == 0


@pytest.mark.parametrize("bad", [0.0, -1.0, math.inf, math.nan])
@pytest.mark.parametrize("room", [1, 80])  # the table's width says how long a sequence may be
def test_forward_unusable_scales_give_zeros(torch, ia, bad, room):
    c = Case(torch, 41, 2, 2, 64, 16, [33, 50], room=room)
    q, s, qt, st = c.queries(torch, 4, 1)
    s[0, 1], s[1, 2] = bad, bad
    got = ia.cache_forward(c.cache, qt, dev(torch, s), dtype=torch.int8)
    assert int((got.cpu().numpy() != plain.attend(q, s, c.k, c.v, c.table, c.lens, c.sk, c.sv)[1]).sum()) == 0
    assert int(got[0, 1].abs().sum()) == 0
    for name in ("sk", "sv"):
        was = getattr(c, name).copy()
        getattr(c, name)[1] = bad
        c.up(torch)
        got = ia.cache_forward(c.cache, qt, st, dtype=torch.float32)
        assert int((got[:, 2:] != 0).sum()) == 0 and int((got[:, :2] != 0).sum()) > 0
        setattr(c, name, was)


@pytest.mark.parametrize("rows, d, page, n", [(16, 64, 16, 2300), (4, 128, 64, 9001), (1, 64, 24, 40000), (33, 128, 128, 2500), (150, 64, 16, 1100), (2, 128, 1, 1030)])
def test_forward_of_long_sequences(torch, ia, rows, d, page, n):
    """Scores past what the kernels keep close by; every key counts."""
    c = Case(torch, rows, 1, 1, d, page, [n], room=0)
    got, wt, want, w = run_forward(torch, ia, c, rows, 1, None)
    check_forward(torch, c, got, wt, want, w, rows, "int8")


@pytest.mark.parametrize("rows, d, page, lens", [(16, 64, 16, [2900, 0, 2112, 2113, 64]), (13, 128, 24, [2600, 2560, 1]), (9, 64, 64, [4800, 3840, 3000]), (4, 64, 16, [2300, 2048, 70, 0]),
                                                  (4, 128, 16, [1500, 900]), (4, 64, 8, [2200, 65]), (2, 64, 64, [4200, 4096, 65]), (16, 128, 64, [2048, 2000, 1]),
                                                  (5, 128, 8, [1030, 64, 0])])
def test_forward_of_long_sequences_among_many_short_ones(torch, ia, rows, d, page, lens):
    """Enough sequences for a workgroup each (176), or more than one to a compute unit (340), and a few of them with more scores than it
    holds."""
    n = 340 if rows <= 4 else 176
    c = Case(torch, rows, n, 1, d, page, lens + [3] * (n - len(lens)), room=0)
    got, wt, want, w = run_forward(torch, ia, c, rows, 1, None)
    check_forward(torch, c, got, wt, want, w, rows, "int8")
    c.table[:len(lens), 1::3] = -1
    c.up(torch)
    got, wt, want, w = run_forward(torch, ia, c, rows, 1, None, weight=False)
    check_forward(torch, c, got, wt, want, w, rows, "int8")


@pytest.mark.parametrize("bits, clip", [(1, 6.6), (3, 5.5), (6, 7.7)])
def test_forward_with_other_tables(torch, bits, clip):
    from paper_2511_21513_amd import binding

    c = Case(torch, bits, 2, 2, 64, 16, [100, 217])
    q, s, qt, st = c.queries(torch, 4, 1)
    other = binding.IntAttn(device=0, lut_bits=bits, clip=clip)
    got = other.cache_forward(c.cache, qt, st, dtype=torch.int8)
    torch.cuda.synchronize()
    other.close()
    assert int((got.cpu().numpy() != plain.attend(q, s, c.k, c.v, c.table, c.lens, c.sk, c.sv, bits=bits, clip=clip)[1]).sum()) == 0


def test_forward_is_the_forward_of_a_contiguous_cache(torch, ia, oracle):
    """The library's own path for one token against contiguous keys, and its oracle: the same bytes."""
    c = Case(torch, 51, 2, 2, 128, 16, [1200, 1200], per_head=True)
    q, s, qt, st = c.queries(torch, 8, 1)
    s[:] = s[0:1, :, :]
    k, v = (np.stack([np.stack([plain.gather(x, c.table[b], 1200, h)[0] for h in range(2)]) for b in range(2)]).astype(np.int8) for x in (c.k, c.v))
    sq = s[0, :, 0].copy()
    got = ia.cache_forward(c.cache, qt, dev(torch, s), dtype=torch.int8).cpu().numpy()
    same = ia.forward(qt, dev(torch, k), dev(torch, v), sq, c.sk, c.sv, None, causal=True, per_head=True).cpu().numpy()
    assert (got == same).all()
    assert (got == oracle.forward(q, k, v, sq, c.sk, c.sv, None, causal=True, per_head=True)["out"]).all()


def test_forward_strides_and_offsets_past_32_bits(torch, ia):
    """A pool whose last pages start past 2^32 bytes, queries and outputs that are views, planes of weights inside larger ones."""
    from paper_2511_21513_amd import binding

    Hkv, d, page, n = 2, 64, 16, 70
    c = Case(torch, 61, 2, Hkv, d, page, [n, 33], spare=2)
    gap = (1 << 32) // (c.n_pages - 1) // 4096 * 4096 + 8192  # bytes between pages
    big = torch.zeros(gap * c.n_pages, dtype=torch.int8, device="cuda")
    kp, vp = (big[o:].as_strided((c.n_pages, Hkv, page, d), (gap, page * 2 * d, 2 * d, 1)) for o in (0, d))  # K and V rows in turn
    kp.copy_(c.t["k"])
    vp.copy_(c.t["v"])
    cache = binding.PagedCache(kp, vp, c.t["table"], c.t["lens"], c.t["sk"], c.t["sv"])
    q, s, qt, st = c.queries(torch, 4, 2)
    qt = qt.transpose(1, 2).contiguous().transpose(1, 2)
    room = torch.full((2, 2, 6, 80), 9, dtype=torch.int8, device="cuda")
    out = room[:, :, 1:5, :64].transpose(1, 2)
    planes = torch.rand((2, 3, Hkv, 100), device="cuda")
    w0 = planes.cpu().numpy().copy()
    got = ia.cache_forward(cache, qt, st, out=out, weight=planes[:, 1], max_len=n)
    torch.cuda.synchronize()
    want = plain.attend(q, s, c.k, c.v, c.table, c.lens, c.sk, c.sv, weight=w0[:, 1])
    assert int((got.cpu().numpy() != want[1]).sum()) == 0
    assert int((room[:, :, 0] != 9).sum()) + int((room[:, :, 5] != 9).sum()) + int((room[..., 64:] != 9).sum()) == 0
    assert (np.abs(wide(planes)[:, 1] - want[3]) <= 8 * 2.0 ** -24 * want[3]).all()
    assert (planes.cpu().numpy()[:, 0::2] == w0[:, 0::2]).all()


# ---------------------------------------------------------------- append

APPENDS = [
    # dtype, B, Hq, Hkv, d, page, L, lens (after), n_new, rot, axes, halves, per_head
    ("float32", 1, 1, 1, 64, 16, 1, [1], None, 64, 1, False, False),
    ("bfloat16", 3, 8, 2, 128, 64, 1, [65, 64, 1], None, 128, 1, False, True),
    ("float16", 2, 4, 4, 64, 16, 20, [50, 20], [20, 7], 64, 3, True, True),
    ("bfloat16", 2, 6, 2, 128, 24, 33, [40, 100], [33, 0], 32, 2, True, False),
    ("float32", 2, 0, 3, 128, 1, 5, [5, 9], None, 128, 1, True, True),
    ("float16", 1, 2, 1, 64, 7, 70, [70], [65], 0, 1, False, True),
    ("float32", 2, 40, 8, 128, 16, 3, [3, 40], [9, -2], 64, 1, False, True),
    ("bfloat16", 1, 2046, 1, 64, 16, 2, [19], None, 64, 1, True, True),         # as many heads as a call may have
    ("float16", 40, 1, 1, 64, 16, 30, [30 + b for b in range(40)], None, 16, 1, False, True),
    ("bfloat16", 30, 2, 2, 128, 8, 70, [70] * 30, [b * 3 for b in range(30)], 128, 2, True, True),
]


@pytest.mark.parametrize("case", APPENDS, ids=str)
def test_append(torch, ia, case):
    dtype, B, Hq, Hkv, d, page, L, lens, n_new, rot, axes, halves, per_head = case
    c = Case(torch, len(str(case)), B, Hkv, d, page, lens, per_head)
    rng = c.rng
    x = [(rng.standard_normal((B, L, max(h, 1), d)) * 1.5).astype(np.float32) for h in (Hq, Hkv, Hkv)]
    q, k, v = (dev(torch, a, dtype).transpose(1, 2) for a in x)
    pos = rng.integers(0, 20000, (axes, B, L)).astype(np.int32)
    freq = 10000.0 ** (-2.0 * np.arange(rot // 2) / max(rot, 1))
    axis = [int(a) for a in rng.integers(0, axes, rot // 2)]
    nn = None if n_new is None else np.array(n_new, dtype=np.int32)
    slots = c.width * page
    weight, order = torch.full((B, Hkv, slots), 3.0, device="cuda"), torch.full((B, Hkv, slots), -9, dtype=torch.int32, device="cuda")
    first = rng.integers(0, 1000, B).astype(np.int32)
    rotary = dict(pos=dev(torch, pos), freq=dev(torch, freq), axis=axis, pairing="halves" if halves else "adjacent") if rot else {}
    got = ia.cache_append(c.cache, k, v, q if Hq else None, n_new=None if nn is None else dev(torch, nn), weight=weight, order=order, first=dev(torch, first), **rotary)
    torch.cuda.synchronize()
    turn = lambda a: plain.turned(a, pos, freq, axis, halves).astype(np.float32) if rot else a.astype(np.float32)
    qx, kx, vx = turn(wide(q)), turn(wide(k)), wide(v).astype(np.float32)
    k_want, v_want = c.k.copy(), c.v.copy()
    w_want, o_want = np.full((B, Hkv, slots), 3.0, np.float32), np.full((B, Hkv, slots), -9, np.int32)
    there = np.zeros((B, L), dtype=bool)
    for b in range(B):
        fresh = min(L, lens[b]) if nn is None else min(max(int(nn[b]), 0), min(L, lens[b]))
        for t in range(fresh):
            there[b, t] = True
            slot = lens[b] - fresh + t
            p, at = c.table[b, slot // page], slot % page
            for h in range(Hkv):
                k_want[p, h, at] = plain.int8(kx[b, h, t], c.sk[h if per_head else 0])
                v_want[p, h, at] = plain.int8(vx[b, h, t], c.sv[h if per_head else 0])
            w_want[b, :, slot], o_want[b, :, slot] = 0.0, first[b] + t
    assert int((c.t["k"].cpu().numpy() != k_want).sum()) == 0 and int((c.t["v"].cpu().numpy() != v_want).sum()) == 0
    assert (weight.cpu().numpy() == w_want).all() and (order.cpu().numpy() == o_want).all()
    if Hq:
        s = (np.maximum(np.abs(qx).max(axis=3), np.float32(1e-12)) / np.float32(127)).astype(np.float32)
        keep = there[:, None, :]
        assert (got[1].cpu().numpy() == np.where(keep, s, 0)).all()
        assert (got[0].cpu().numpy() == np.where(keep[..., None], plain.int8(qx, s[..., None]), 0)).all()


def test_append_leaves_absent_pages_alone_and_stays_inside_the_table(torch, ia):
    c = Case(torch, 71, 3, 2, 64, 16, [40, 40, 40], room=0)
    c.table[0, 2], c.table[1, 1] = -1, c.n_pages
    c.lens = np.array([40, 40, 10 ** 9], dtype=np.int32)  # the last: 48 slots
    c.up(torch)
    x = torch.randn((3, 2, 30, 64), device="cuda")
    ia.cache_append(c.cache, x, x)
    torch.cuda.synchronize()
    k_want = c.k.copy()
    for b, n in enumerate((40, 40, 48)):
        for t in range(30):
            p = plain.page_of(c.table[b], n - 30 + t, 16, c.n_pages)
            if p is not None:
                for h in range(2):
                    k_want[p, h, (n - 30 + t) % 16] = plain.int8(x[b, h, t].cpu().numpy(), c.sk[h])
    assert int((c.t["k"].cpu().numpy() != k_want).sum()) == 0


def test_new_outputs_of_broadcast_inputs(torch, ia):
    """Inputs with axes of stride 0, and with axes of one element of any stride."""
    c = Case(torch, 73, 2, 2, 64, 16, [40, 33])
    x = torch.randn((1, 1, 1, 64), device="cuda", dtype=torch.bfloat16)
    pos, freq = torch.arange(3, device="cuda", dtype=torch.int32).expand(1, 2, 3), torch.rand(32, device="cuda", dtype=torch.float64)
    whole = lambda t: t.contiguous()
    for q in (x.expand(2, 4, 3, 64), x.expand(2, 4, 1, 64).contiguous().expand(2, 4, 3, 64), torch.randn((2, 3, 4, 64), device="cuda", dtype=torch.bfloat16).transpose(1, 2)):
        assert torch.equal(ia.rope(q, pos, freq), ia.rope(whole(q), pos, freq))
        k = q[:, :2]
        (a, sa), (b, sb) = ia.cache_append(c.cache, k, k, q), ia.cache_append(c.cache, whole(k), whole(k), whole(q))
        assert torch.equal(a, b) and torch.equal(sa, sb)
        q8 = a[:1, :, :1].expand(2, 4, 3, 64)
        assert torch.equal(ia.cache_forward(c.cache, q8, sa), ia.cache_forward(c.cache, whole(q8), sa))
    one = torch.randn((2 * 4 * 64 + 8,), device="cuda", dtype=torch.bfloat16).as_strided((2, 4, 1, 64), (256, 64, 8, 1))
    (a, sa), (b, sb) = ia.cache_append(c.cache, one[:, :2], one[:, :2], one), ia.cache_append(c.cache, whole(one[:, :2]), whole(one[:, :2]), whole(one))
    assert torch.equal(a, b) and torch.equal(sa, sb)


@pytest.mark.parametrize("scale", [1e-45, 3e-41, 2.0 ** -126, 2.0 ** -101, 1e-30, 2.0 ** 101, 1e38, 3.4e38])
def test_append_at_scales_of_all_sizes(torch, ia, scale):
    """Subnormal scales, scales whose reciprocal is subnormal, and elements on and beside the ties."""
    c = Case(torch, 72, 1, 2, 64, 16, [33], room=0)
    s = np.float32(scale)
    c.sk[:], c.sv[:] = s, s
    c.up(torch)
    ratio = c.rng.integers(-260, 261, (1, 2, 33, 64)) / 2.0
    with np.errstate(over="ignore"):
        x = (ratio * np.float64(s)).astype(np.float32)
    x = np.where(np.isfinite(x), x, np.float32(3.4e38) * np.sign(ratio).astype(np.float32)).astype(np.float32)
    near = c.rng.random(x.shape)
    x = np.where(near < 0.2, np.nextafter(x, np.float32(0)), x).astype(np.float32)
    ia.cache_append(c.cache, dev(torch, x), dev(torch, -x))
    torch.cuda.synchronize()
    k, v = c.t["k"].cpu().numpy(), c.t["v"].cpu().numpy()
    for h in range(2):
        for t in range(33):
            page, at = c.table[0, t // 16], t % 16
            assert (k[page, h, at] == plain.int8(x[0, h, t], s)).all() and (v[page, h, at] == plain.int8(-x[0, h, t], s)).all()


def test_append_is_rope_and_the_quantizer(torch, ia):
    """The same integers as the library's separate operators give: rope in 32 bits, then a scale for each token."""
    xs, pos, freq, axis = rope_case(8, 2, 21, (4, 2), 64, 64, 2, 8000)
    c = Case(torch, 81, 2, 2, 64, 16, [21, 60])
    q, k = (dev(torch, x) for x in xs)
    p, f = dev(torch, pos), dev(torch, freq)
    q8, qs = ia.cache_append(c.cache, k, k, q, pos=p, freq=f, axis=axis)
    want, scales = ia.quantize(ia.rope(q, p, f, axis=axis), q_block=1)
    torch.cuda.synchronize()
    assert torch.equal(q8, want) and torch.equal(qs, scales)


# ---------------------------------------------------------------- eviction

EVICTS = [
    # B, Hkv, d, page, lens, keep, sink, recent, how
    (1, 1, 64, 16, [2], 1, 0, 0, "plain"),
    (3, 2, 64, 16, [100, 64, 10], 64, 4, 8, "plain"),
    (2, 4, 128, 24, [500, 333], 200, 0, 50, "equal"),
    (2, 2, 64, 1, [90, 41], 40, 2, 3, "plain"),
    (2, 2, 128, 64, [1500, 1100], 1050, 10, 900, "held"),   # more keys are held than stay
    (2, 2, 64, 16, [3000, 2048], 1024, 4, 64, "zeros"),
    (1, 3, 64, 16, [700], 350, 0, 0, "odd"),                # infinities, NaN, both zeros, negative
    (2, 2, 64, 16, [130, 200], 100, 3, 9, "slots"),         # no orders: the slot counts
    (1, 2, 64, 32, [5000], 4999, 1, 1, "equal"),
    (1, 1, 64, 16, [20000], 9000, 4, 500, "plain"),
    (1, 2, 64, 16, [900], 450, 0, 0, "wide"),               # weights of all exponents
    (2, 1, 64, 16, [1300, 700], 600, 0, 0, "narrow"),       # of three values next to each other, order by order
    (1, 2, 64, 16, [18000], 700, 3, 900, "held"),
    (1, 1, 64, 16, [26000], 9000, 4, 500, "plain"),         # more keys than registers hold
    (2, 1, 64, 16, [25000, 4000], 24000, 4, 64, "zeros"),
    (270, 1, 64, 16, [5000, 4999, 4097] + [20] * 267, 4096, 2, 64, "equal"),  # workgroups of half the size
    (300, 1, 64, 64, [12000, 11000, 90] + [1] * 297, 80, 2, 20, "plain"),
]


@pytest.mark.parametrize("place", ["in place", "elsewhere"])
@pytest.mark.parametrize("case", EVICTS, ids=lambda c: str(c)[:60])
def test_evict(torch, ia, case, place):
    B, Hkv, d, page, lens, keep, sink, recent, how = case
    c = Case(torch, len(str(case)), B, Hkv, d, page, lens)
    rng, slots = c.rng, c.width * page
    w = rng.random((B, Hkv, slots)).astype(np.float32)
    if how == "equal":
        w = (w * 4).astype(np.int32).astype(np.float32)
    if how == "zeros":
        w = np.where(rng.random(w.shape) < 0.7, 0, w).astype(np.float32)
    if how == "wide":
        w = (2.0 ** rng.uniform(-148, 127, w.shape)).astype(np.float32)
    if how == "narrow":
        w = (np.float32(0.3) + rng.integers(0, 3, w.shape) * np.float32(2.0 ** -25)).astype(np.float32)
    if how == "odd":
        odd = np.array([np.inf, -np.inf, np.nan, -np.nan, 0.0, -0.0, -1.5, 3e38, 1e-45], dtype=np.float32)
        w = np.where(rng.random(w.shape) < 0.5, odd[rng.integers(0, 9, w.shape)], w).astype(np.float32)
    order = None if how == "slots" else np.argsort(rng.random((B, Hkv, slots)), axis=2).astype(np.int32)
    if how == "odd":
        order = rng.integers(0, 5, order.shape).astype(np.int32)
    total = np.array(lens, dtype=np.int32) if how != "held" else np.full(B, slots, np.int32)
    before = plain.evict(c.k, c.v, c.table, c.lens, w, order, keep, total, sink, recent)
    wt, ot, tt = dev(torch, w), None if order is None else dev(torch, order), dev(torch, total)
    outs = {}
    if place == "elsewhere":
        outs = dict(weight_out=torch.full_like(wt, -5), lens_out=torch.zeros_like(c.t["lens"]), order_out=None if order is None else torch.full_like(ot, -5))
    ia.cache_evict(c.cache, keep, wt, order=ot, total=tt, sink=sink, recent=recent, **outs)
    torch.cuda.synchronize()
    k_want, v_want, w_want, o_want, n_want = before
    assert int((c.t["k"].cpu().numpy() != k_want).sum()) == 0 and int((c.t["v"].cpu().numpy() != v_want).sum()) == 0
    got_n = outs.get("lens_out", c.t["lens"]).cpu().numpy()
    assert (got_n == n_want).all()
    under = np.arange(slots)[None, None] < n_want[:, None, None]
    got_w = outs.get("weight_out", wt).cpu().numpy()
    same = (got_w.view(np.int32) == np.where(under, w_want, w if place == "in place" else np.float32(-5)).astype(np.float32).view(np.int32))
    assert same.all()
    if order is not None:
        got_o = (outs["order_out"] if outs else ot).cpu().numpy()
        assert (got_o == np.where(under, o_want, order if place == "in place" else -5)).all()
    if place == "elsewhere":
        assert (wt.cpu().numpy().view(np.int32) == w.view(np.int32)).all() and (c.t["lens"].cpu().numpy() == np.array(lens)).all()


def test_evict_leaves_sequences_with_absent_pages_alone(torch, ia):
    c = Case(torch, 91, 3, 2, 64, 16, [100, 100, 100])
    c.table[1, 3], c.table[2, -1] = -1, -1  # the last is behind the end of its sequence
    c.up(torch)
    w = c.rng.random((3, 2, c.width * 16)).astype(np.float32)
    want = plain.evict(c.k, c.v, c.table, c.lens, w, None, 40)
    wt = dev(torch, w)
    ia.cache_evict(c.cache, 40, wt)
    torch.cuda.synchronize()
    assert c.t["lens"].cpu().numpy().tolist() == want[4].tolist() == [40, 100, 40]
    assert int((c.t["k"].cpu().numpy() != want[0]).sum()) == 0
    assert (wt.cpu().numpy()[1] == w[1]).all()


# ---------------------------------------------------------------- together, streams, graphs

def serve(torch, ia, steps, stream=None):
    """A few steps of serving two sequences: append with rotation, attend with weights, evict to a budget; the plain forms step beside."""
    c = Case(torch, 101, 2, 2, 64, 16, [70, 41], room=3)
    rng, Hq, slots = c.rng, 4, c.width * 16
    w, order = np.zeros((2, 2, slots), np.float32), np.tile(np.arange(slots, dtype=np.int32), (2, 2, 1))
    wt, ot = dev(torch, w), dev(torch, order)
    k, v, lens, total = c.k, c.v, c.lens.copy(), c.lens.copy()
    w = w.astype(np.float64)
    freq = 10000.0 ** (-2.0 * np.arange(32) / 64)
    ft, tt = dev(torch, freq), dev(torch, total)
    for step in range(steps):
        L = (1, 3, 1, 2)[step % 4]
        n_new = np.array([L, max(1, L - 1)], dtype=np.int32)
        x = [rng.standard_normal((2, h, L, 64)).astype(np.float32) for h in (Hq, 2, 2)]
        pos = (total[:, None] + np.arange(L)).astype(np.int32)[None]
        first, lens, total = total.copy(), lens + n_new, total + n_new
        c.t["lens"].copy_(dev(torch, lens))
        q8, qs = ia.cache_append(c.cache, dev(torch, x[1]), dev(torch, x[2]), dev(torch, x[0]), n_new=dev(torch, n_new), pos=dev(torch, pos), freq=ft, weight=wt, order=ot,
                                 first=dev(torch, first))
        out = ia.cache_forward(c.cache, q8, qs, dtype=torch.int8, n_new=dev(torch, n_new), weight=wt, decay=0.9)
        tt.copy_(dev(torch, total))
        if step % 3 == 2:
            ia.cache_evict(c.cache, 60, wt, order=ot, total=tt, sink=2, recent=16)
        torch.cuda.synchronize()
        # beside
        turned = [plain.turned(a, pos, freq, [0] * 32, False).astype(np.float32) for a in x[:2]]
        sq = (np.abs(turned[0]).max(axis=3) / np.float32(127)).astype(np.float32)
        q = plain.int8(turned[0], sq[..., None])
        for b in range(2):
            for t in range(n_new[b]):
                slot = lens[b] - n_new[b] + t
                for h in range(2):
                    k[c.table[b, slot // 16], h, slot % 16] = plain.int8(turned[1][b, h, t], c.sk[h])
                    v[c.table[b, slot // 16], h, slot % 16] = plain.int8(x[2][b, h, t], c.sv[h])
                w[b, :, slot], order[b, :, slot] = 0, first[b] + t
            q[b, :, n_new[b]:], sq[b, :, n_new[b]:] = 0, 0
        _, out8, _, w = plain.attend(q, sq, k, v, c.table, lens, c.sk, c.sv, n_new=n_new, weight=w, decay=np.float32(0.9))
        assert int((out.cpu().numpy() != out8).sum()) == 0, f"step {step}"
        if step % 3 == 2:
            w32 = wt_before_evict = w.astype(np.float32)
            k, v, w, order, lens = plain.evict(k, v, c.table, lens, w32, order, 60, total, 2, 16)
            w = w.astype(np.float64)
        assert (c.t["lens"].cpu().numpy() == lens).all()
        assert int((c.t["k"].cpu().numpy() != k).sum()) == 0 and int((c.t["v"].cpu().numpy() != v).sum()) == 0, f"step {step}"
        for b in range(2):
            assert np.allclose(wide(wt)[b, :, :lens[b]], w[b, :, :lens[b]], rtol=40 * 2.0 ** -24 * (step + 1), atol=0)
            assert (ot.cpu().numpy()[b, :, :lens[b]] == order[b, :, :lens[b]]).all()


def test_serving_steps(torch, ia):
    serve(torch, ia, 8)


def test_serving_steps_on_another_stream(torch, ia):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        serve(torch, ia, 4)
    torch.cuda.synchronize()


def test_captured_step_replays_with_new_lengths(torch):
    """Append, attention and eviction in one graph: each replay sees the lengths, inputs and tables of its time, with eager work between."""
    from paper_2511_21513_amd import binding

    ia, other = binding.IntAttn(device=0), binding.IntAttn(device=0)
    B, Hkv, Hq, d, page = 2, 2, 8, 64, 16
    c = Case(torch, 111, B, Hkv, d, page, [3000, 3000], room=1)  # long enough that scores leave the workgroup
    slots = c.width * page
    q, k, v = (torch.randn((B, h, 1, d), device="cuda") for h in (Hq, Hkv, Hkv))
    pos, freq = torch.zeros((1, B, 1), dtype=torch.int32, device="cuda"), dev(torch, 10000.0 ** (-np.arange(32) / 32))
    w, out = torch.rand((B, Hkv, slots), device="cuda"), torch.empty((B, Hq, 1, d), dtype=torch.int8, device="cuda")
    w2, n2 = torch.empty_like(w), torch.empty_like(c.t["lens"])
    q8, qs = torch.empty((B, Hq, 1, d), dtype=torch.int8, device="cuda"), torch.empty((B, Hq, 1), device="cuda")

    def step():
        ia.cache_append(c.cache, k, v, q, pos=pos, freq=freq, q_out=q8, q_scale=qs)
        ia.cache_forward(c.cache, q8, qs, out=out, weight=w)
        ia.cache_evict(c.cache, 1500, w, weight_out=w2, lens_out=n2)

    ia.cache_reserve(c.cache, rows=Hq // Hkv, keep=1500)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step()
    for n in ([2999, 1], [700, 1600], [64, 3001]):
        c.t["lens"].copy_(dev(torch, np.array(n, dtype=np.int32)))
        q.copy_(torch.randn_like(q))
        pos.fill_(n[0])
        state = [x.clone() for x in (c.t["k"], c.t["v"], w)]
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, w, w2[:, :, :1], n2, c.t["k"], c.t["v"])]
        for x, y in zip((c.t["k"], c.t["v"], w), state):
            x.copy_(y)
        ia, keep = other, ia  # the same, eagerly and from another context
        step()
        torch.cuda.synchronize()
        ia = keep
        for x, y in zip(got, (out, w, w2[:, :, :1], n2, c.t["k"], c.t["v"])):
            assert torch.equal(x, y)
    other.close()
    ia.close()


@pytest.mark.parametrize("d, page, most", [(64, 16, 250), (128, 8, 200), (128, 32, 60)])
def test_forward_of_very_many_short_sequences(torch, ia, d, page, most):
    c = Case(torch, d + most, 800, 2, d, page, [i % (most + 1) for i in range(799)] + [most], room=0)
    got, wt, want, w = run_forward(torch, ia, c, 6, 1, None)
    check_forward(torch, c, got, wt, want, w, 3, "int8")


@pytest.mark.parametrize("weight", [False, True])
def test_forward_of_as_many_rows_as_a_call_may_have(torch, ia, weight):
    c = Case(torch, 131, 2, 1, 64, 16, [700, 64], room=0)
    got, wt, want, w = run_forward(torch, ia, c, 64, 64, [64, 33], weight=weight)
    check_forward(torch, c, got, wt, want, w, 4096, "int8")


def test_graphs_keep_their_room_when_it_is_outgrown(torch):
    """Two graphs on one context, and an eager call in between that needs more room than the first was captured with."""
    from paper_2511_21513_amd import binding

    own = binding.IntAttn(device=0)
    cases = []
    for i, (n, rows) in enumerate(((2600, 4), (9000, 20))):
        c = Case(torch, 141 + i, 1, 2, 64, 16, [n], room=0)
        q, s, qt, st = c.queries(torch, 2 * rows, 1)
        w0 = torch.rand((1, 2, c.width * 16), device="cuda")
        w, out = torch.empty_like(w0), torch.empty((1, 2 * rows, 1, 64), dtype=torch.int8, device="cuda")
        own.cache_forward(c.cache, qt, st, out=out, weight=w0, weight_out=w)  # grows the room
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            own.cache_forward(c.cache, qt, st, out=out, weight=w0, weight_out=w)
        acc, want, real, new = plain.attend(q, s, c.k, c.v, c.table, c.lens, c.sk, c.sv, weight=w0.cpu().numpy())
        cases.append((c, graph, out, w, want, new, rows, qt, st, w0))  # (what a graph reads has to live)
    for turn in range(3):
        for c, graph, out, w, want, new, rows, qt, st, w0 in cases:
            out.fill_(5)
            w.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert int((out.cpu().numpy() != want).sum()) == 0
            assert (np.abs(wide(w) - new)[..., :c.lens[0]] <= (rows + 3) * 2.0 ** -24 * new[..., :c.lens[0]]).all()
        out = own.cache_forward(cases[turn % 2][0].cache, cases[turn % 2][7], cases[turn % 2][8], dtype=torch.int8)
        assert int((out.cpu().numpy() != cases[turn % 2][4]).sum()) == 0
    del cases, graph
    own.close()


def test_room_is_reserved_for_fewer_rows_too(torch):
    """The kernels that a call takes depend on its rows and on whether weights are kept; a reservation holds for all of them."""
    from paper_2511_21513_amd import binding

    own = binding.IntAttn(device=0)
    c = Case(torch, 121, 1, 2, 64, 16, [2600], room=0)
    own.cache_reserve(c.cache, rows=40)
    for rows, L in ((1, 1), (4, 1), (16, 1), (5, 4), (20, 2), (40, 1)):
        for weight in (False, True):
            q, s, qt, st = c.queries(torch, 2 * rows, L) if rows * L <= 40 else (None,) * 4
            if q is None:
                continue
            w = torch.rand((1, 2, c.width * 16), device="cuda") if weight else None
            out, stream = torch.empty((1, 2 * rows, L, 64), dtype=torch.int8, device="cuda"), torch.cuda.Stream()
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=stream):
                own.cache_forward(c.cache, qt, st, out=out, weight=w)
            want = plain.attend(q, s, c.k, c.v, c.table, c.lens, c.sk, c.sv)[1]
            for _ in range(3):
                out.fill_(77)
                graph.replay()
                torch.cuda.synchronize()
                assert int((out.cpu().numpy() != want).sum()) == 0
            del graph
    own.close()


def test_a_captured_call_without_room_is_refused(torch):
    from paper_2511_21513_amd import binding

    ia = binding.IntAttn(device=0)
    c = Case(torch, 121, 1, 1, 64, 16, [40], room=0)
    w = torch.rand((1, 1, 48), device="cuda")
    x = torch.zeros(4, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        x += 1
        with pytest.raises(binding.IntAttnError) as e:
            ia.cache_evict(c.cache, 20, w)
        assert e.value.code == binding.ERR_NOMEM and "cache_reserve" in str(e.value)
    graph.replay()
    ia.cache_evict(c.cache, 20, w)
    torch.cuda.synchronize()
    assert int(c.t["lens"][0]) == 20 and float(x[0]) == 1.0
    ia.close()


def test_binding_refuses_what_pointers_do_not_carry(torch, ia):
    from paper_2511_21513_amd import binding

    c = Case(torch, 131, 2, 2, 64, 16, [20, 30])
    q, s, qt, st = c.queries(torch, 4, 1)
    t = c.t
    for make in (lambda: binding.PagedCache(t["k"].float(), t["v"], t["table"], t["lens"], t["sk"], t["sv"]),
                 lambda: binding.PagedCache(t["k"], t["v"][:, :1], t["table"], t["lens"], t["sk"], t["sv"]),
                 lambda: binding.PagedCache(t["k"], t["v"], t["table"].long(), t["lens"], t["sk"], t["sv"]),
                 lambda: binding.PagedCache(t["k"], t["v"], t["table"], t["lens"][:1], t["sk"], t["sv"]),
                 lambda: binding.PagedCache(t["k"], t["v"], t["table"], t["lens"].cpu(), t["sk"], t["sv"]),
                 lambda: binding.PagedCache(t["k"], t["v"], t["table"], t["lens"], t["sk"], t["sv"][:1]),
                 lambda: ia.cache_forward(c.cache, qt[:, :3], st[:, :3]), lambda: ia.cache_forward(c.cache, qt, st.double()),
                 lambda: ia.cache_forward(c.cache, qt, st[..., :0]), lambda: ia.cache_forward(c.cache, qt, st, dtype=torch.float64),
                 lambda: ia.cache_forward(c.cache, qt, st, weight=torch.zeros((2, 2, 16), device="cuda")),
                 lambda: ia.cache_append(c.cache, qt.float()[:, :2], qt.half()[:, :2]), lambda: ia.cache_append(c.cache, qt[:, :2], qt[:, :2]),
                 lambda: ia.cache_evict(c.cache, 5, torch.zeros((2, 2, 20), device="cuda")),
                 lambda: ia.rope(qt.float(), torch.zeros((2, 1), dtype=torch.int32, device="cuda"), torch.ones(32, device="cuda")),
                 lambda: ia.rope(qt.float(), torch.zeros((2, 1), dtype=torch.int32, device="cuda"), torch.ones(32, device="cuda", dtype=torch.float64), axis=[0] * 31)):
        with pytest.raises((ValueError, binding.IntAttnError)):
            make()
