"""The operators around a paged INT8 key/value cache, as cases that can be timed and compared.

What a serving program does with such a cache, each through the public binding:
  rope     rotary positions with several axes on Q and K (prefill, images and video, and the gradient: the inverse rotation)
  append   new tokens' K rotated, K and V quantized into their pages, Q rotated and quantized per token
  attend   attention of one new token (or a few) over the pages: INT8 Q.K^T, IndexSoftmax, P.V, and the attention weight that
           each cached key has drawn so far
  evict    the keys that drew least leave the cache, the others are moved together
Without the library's kernels the same is computed with elementary torch operations.

The integers are defined exactly.  A rotated channel is the 32-bit rounding of the rotation in real numbers; the scale of a row
is fl32(max|x| / 127) and its integers are rint(fl32(x / scale)), ties to even, clamped to 127.  Attention is the library's
integer pipeline: c_int = floor(clip sqrt(d) / (s_q s_k) + 1/2), index = round-half-up((2^b - 1) min(max - A, c_int) / c_int),
E = table[index], P = round-half-up(255 E / sum E), output = (P.V) s_v / 255, or with an output scale the INT8 requantization.
"""
import math

import numpy as np
import torch

own = False

CLIP = 6.6  # the library's default clip bound, and 2^5 table entries
TOP = 31

DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16, "int8": torch.int8}


def listed():
    return [
        # one new token for each of 8 conversations: the smallest call, where the launch counts
        dict(name="rope_token_b8", op="rope", B=8, L=1, Hq=32, Hkv=8, d=128, rot=128, axes=1, pairing="adjacent", inverse=False, dtype="bfloat16", far=100000),
        # a prompt of image patches and text: positions in time, height and width, channels in halves, a ragged length
        dict(name="rope_image_2x1531", op="rope", B=2, L=1531, Hq=16, Hkv=16, d=64, rot=64, axes=3, pairing="halves", inverse=False, dtype="float16", far=4096),
        # the gradient of a long training sequence: the inverse rotation, in 32 bits
        dict(name="rope_gradient_8k", op="rope", B=1, L=8192, Hq=32, Hkv=8, d=128, rot=128, axes=1, pairing="adjacent", inverse=True, dtype="float32", far=8192),
        # one new token for each of 32 conversations: what every layer of a decoding step starts with
        dict(name="append_token_b32", op="append", B=32, L=1, Hq=32, Hkv=8, d=128, page=64, lo=500, hi=1700, rot=128, axes=1, pairing="adjacent", dtype="bfloat16", per_head=True),
        # two padded prompts with image positions into pages of 16
        dict(name="append_prompt_2x1021", op="append", B=2, L=1021, Hq=16, Hkv=16, d=64, page=16, lo=700, hi=1021, rot=64, axes=3, pairing="halves", dtype="float16", per_head=False),
        # a long prompt
        dict(name="append_prompt_8k", op="append", B=1, L=8192, Hq=32, Hkv=8, d=128, page=64, lo=8192, hi=8192, rot=128, axes=1, pairing="adjacent", dtype="bfloat16", per_head=True),
        # a single conversation, at its beginning and far into a long document
        dict(name="attend_b1_700", op="attend", B=1, L=1, Hq=32, Hkv=8, d=128, page=64, lo=700, hi=700, dtype="bfloat16", per_head=True, weight=False),
        dict(name="attend_b1_30011", op="attend", B=1, L=1, Hq=32, Hkv=8, d=128, page=64, lo=30011, hi=30011, dtype="bfloat16", per_head=True, weight=True),
        # many conversations of different lengths: bound by the cache; the weights of the keys are kept for eviction
        dict(name="attend_b32_ragged", op="attend", B=32, L=1, Hq=32, Hkv=8, d=128, page=64, lo=4000, hi=12400, dtype="bfloat16", per_head=True, weight=True),
        # one head of keys for each query head, small pages, up to three drafted tokens checked at once (fewer for some), INT8 output
        dict(name="attend_draft_b16", op="attend", B=16, L=3, Hq=16, Hkv=16, d=64, page=16, lo=100, hi=3900, dtype="int8", per_head=False, weight=False),
        # a page's worth of keys leaves every head of a few conversations
        dict(name="evict_b4_1k", op="evict", B=4, Hkv=8, d=128, page=64, lo=1100, hi=1152, keep=1088, sink=4, recent=64),
        # caches of many conversations cut to a budget
        dict(name="evict_b16_8k", op="evict", B=16, Hkv=8, d=128, page=64, lo=7000, hi=10001, keep=6144, sink=4, recent=512),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(1, 1), (8, 8), (16, 16), (12, 4), (16, 2), (32, 8), (32, 32), (28, 4), (32, 1), (40, 8)]


def draw(rng):
    """One more case of the ranges above: sizes over their whole range, and no more bytes than the largest listed case of its kind."""
    while True:
        op = rng.choice(["rope", "append", "attend", "attend", "attend", "evict"])
        hq, hkv = rng.choice(HEADS)
        d = rng.choice([64, 128])
        page = rng.choice([1, 8, 16, 16, 24, 32, 64, 64, 100, 128, 256])
        axes = rng.choice([1, 1, 2, 3])
        rot = rng.choice([d, d, d // 2, d // 4])
        pairing = rng.choice(["adjacent", "halves"])
        dtype = rng.choice(["float32", "float16", "bfloat16"])
        if op == "rope":
            c = dict(op=op, B=_log_int(rng, 1, 64), L=_log_int(rng, 1, 9000), Hq=hq, Hkv=hkv, d=d, rot=rot, axes=axes, pairing=pairing,
                     inverse=rng.random() < 0.5, dtype=dtype, far=_log_int(rng, 2000, 1000000))
            most = 8192 * 40 * 128 * 8
        elif op == "append":
            L = _log_int(rng, 1, 9000)
            before = 0 if L > 1 and rng.random() < 0.5 else _log_int(rng, 1, 4000)
            c = dict(op=op, B=_log_int(rng, 1, 64), L=L, Hq=hq, Hkv=hkv, d=d, page=page, lo=max(1, before + L // 2), hi=before + L, rot=rng.choice([0, rot, rot]),
                     axes=axes, pairing=pairing, dtype=dtype, per_head=rng.random() < 0.5)
            most = 8192 * 48 * 128 * 3
        elif op == "attend":
            hi = _log_int(rng, 1, 33000)
            c = dict(op=op, B=_log_int(rng, 1, 64), L=rng.choice([1, 1, 1, 1, 2, 4, 7]), Hq=hq, Hkv=hkv, d=d, page=page, lo=rng.choice([hi, max(1, hi // 3), 1]), hi=hi,
                     dtype=rng.choice([dtype, dtype, "int8"]), per_head=rng.random() < 0.5, weight=rng.random() < 0.5)
            most = 32 * 8 * 8192 * 256
        else:
            hi = _log_int(rng, 8, 20000)
            c = dict(op=op, B=_log_int(rng, 1, 32), Hkv=hkv, d=d, page=page, lo=rng.choice([hi, max(1, hi // 2)]), hi=hi)
            c["keep"] = max(1, int(hi * rng.choice([0.5, 0.75, 0.97])))
            c["sink"] = min(4, c["keep"] // 2)
            c["recent"] = min(_log_int(rng, 1, 600), c["keep"] - c["sink"])
            most = 16 * 8 * 3000 * 600
        pool = c["B"] * hkv * c.get("hi", 1) * d * 2
        if work(c)["bytes"] <= most and pool <= 1 << 30:
            return c


def _lens(case):
    """Lengths of the sequences, spread evenly over lo .. hi in an order that is not sorted."""
    b = torch.arange(case["B"], dtype=torch.float64)
    u = (b * 0.6180339887498949 + 0.999) % 1.0
    n = case["lo"] + torch.floor((case["hi"] - case["lo"] + 1) * u).to(torch.int64)
    return n.clamp(max=case["hi"]).to(torch.int32)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _frequencies(rot):
    """Radians per position of each rotated pair: 10000^(-2 i / rot)."""
    return 10000.0 ** (-2.0 * torch.arange(rot // 2, device="cuda", dtype=torch.float64) / rot)


def _positions(case, g):
    """[axes, B, L]: text counts up from an offset; images have a row and a column of a grid as well."""
    B, L, axes = case["B"], case["L"], case["axes"]
    t = torch.arange(L, device="cuda", dtype=torch.int64)[None, :]
    far = case.get("far", case.get("hi", 0))
    first = torch.randint(0, max(1, far - L), (B, 1), generator=g, device="cuda")
    planes = [first + (t if axes == 1 else t // 196), first + t % 196 // 14, first + t % 14]
    return torch.stack([p.expand(B, L) for p in planes[:axes]]).to(torch.int32).contiguous()


def _axis_of_pair(case):
    """Axis that turns each pair: the pairs in equal runs, the first axis takes what is left over."""
    n, axes = case["rot"] // 2, case["axes"]
    run = n // axes
    return [max(0, axes - 1 - (n - 1 - i) // run) if axes > 1 and run else 0 for i in range(n)]


def _pages(case, g, lens, hot=9.0):
    """A pool of pages with keys and values, the table of each sequence's pages (in no order), and the scales."""
    B, Hkv, d, page = case["B"], case["Hkv"], case["d"], case["page"]
    width = -(-int(case["hi"]) // page) + 1
    n_pages = B * width + 3
    table = torch.randperm(n_pages, generator=g, device="cuda")[:B * width].reshape(B, width).to(torch.int32)
    k, v = (torch.empty((n_pages, Hkv, page, d), dtype=torch.int8, device="cuda") for _ in range(2))
    k.random_(-64, 65, generator=g)
    v.random_(-127, 128, generator=g)
    channel = torch.randint(0, d, (Hkv,), generator=g, device="cuda")
    k[:, torch.arange(Hkv, device="cuda"), :, channel] = torch.randint(-127, 128, (Hkv, n_pages, page), generator=g, device="cuda").to(torch.int8)
    n = Hkv if case.get("per_head", True) else 1
    scale_k = (0.02 + 0.01 * torch.rand(n, generator=g, device="cuda")).float()
    scale_v = (0.02 + 0.01 * torch.rand(n, generator=g, device="cuda")).float()
    return k, v, table, lens.cuda(), scale_k, scale_v


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    if case["op"] == "rope":
        dtype = DTYPES[case["dtype"]]
        s["q"], s["k"] = (_normal(g, case["B"], case["L"], h, case["d"]).to(dtype).transpose(1, 2) for h in (case["Hq"], case["Hkv"]))
        s["pos"], s["freq"], s["axis"] = _positions(case, g), _frequencies(case["rot"]), _axis_of_pair(case)
        s["axis_dev"] = torch.tensor(s["axis"], device="cuda")
        return s
    lens = _lens(case)
    s["k_pages"], s["v_pages"], s["table"], s["lens"], s["scale_k"], s["scale_v"] = _pages(case, g, lens)
    B, Hkv, d, hi = case["B"], case["Hkv"], case["d"], case["hi"]
    if case["op"] == "append":
        dtype, L = DTYPES[case["dtype"]], case["L"]
        # projections give [B, L, heads, d]
        s["q"], s["k"], s["v"] = (_normal(g, B, L, h, d).to(dtype).transpose(1, 2) for h in (case["Hq"], Hkv, Hkv))
        s["n_new"] = torch.minimum(s["lens"], torch.full_like(s["lens"], L))
        s["pos"], s["freq"], s["axis"] = _positions(case, g), _frequencies(case["rot"]), _axis_of_pair(case)
        s["axis_dev"] = torch.tensor(s["axis"], device="cuda", dtype=torch.int64)
    elif case["op"] == "attend":
        Hq, L = case["Hq"], case["L"]
        q = 2.5 * _normal(g, B, Hq, L, d)
        q[:, :, :, 0] *= 3.0
        s["scale_q"] = (q.abs().amax(dim=3).double() / 127).float()
        s["q"] = torch.round((q.double() / s["scale_q"].double()[..., None]).float()).clamp_(-127, 127).to(torch.int8)
        s["n_new"] = torch.minimum(s["lens"], torch.randint(1, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32))
        s["scale_out"] = (0.01 + 0.01 * torch.rand(Hq if case["per_head"] else 1, generator=g, device="cuda")).float()
        if case["weight"]:
            s["weight"] = torch.rand((B, Hkv, hi), generator=g, device="cuda") ** 4
            s["weight_out"] = s["weight"].clone()
    else:
        # weights as softmax rows add up: many keys next to nothing (some exactly nothing), few a lot
        w = torch.rand((B, Hkv, hi), generator=g, device="cuda") ** 6 * 3
        s["weight"] = torch.where(w < 1e-4, torch.zeros_like(w), w)
        s["order"] = torch.argsort(torch.rand((B, Hkv, hi), generator=g, device="cuda"), dim=2).to(torch.int32)
        s["total"] = torch.full((B,), hi, dtype=torch.int32, device="cuda")
        s["weight_out"], s["order_out"], s["lens_out"] = s["weight"].clone(), s["order"].clone(), s["lens"].clone()
    return s


# ---------------------------------------------------------------- the library's kernels

_kept = {}


def _context():
    """The program's one context."""
    if "ia" not in _kept:
        from paper_2511_21513_amd import binding

        _kept["ia"] = binding.IntAttn()
    return _kept["ia"]


def _cache(s):
    """The program's handle of its cache."""
    if "cache" not in s:
        from paper_2511_21513_amd import binding

        s["cache"] = binding.PagedCache(s["k_pages"], s["v_pages"], s["table"], s["lens"], s["scale_k"], s["scale_v"])
    return s["cache"]


def _run_own(s):
    case, ia = s["case"], _context()
    if case["op"] == "rope":
        q, k = ia.rope([s["q"], s["k"]], s["pos"], s["freq"], axis=s["axis"], pairing=case["pairing"], inverse=case["inverse"])
        return dict(q=q, k=k)
    if case["op"] == "append":
        rotary = dict(pos=s["pos"], freq=s["freq"], axis=s["axis"], pairing=case["pairing"]) if case["rot"] else {}
        q, scale_q = ia.cache_append(_cache(s), s["k"], s["v"], s["q"], n_new=s["n_new"], **rotary)
        return dict(q=q, scale_q=scale_q, k_pages=s["k_pages"], v_pages=s["v_pages"])
    if case["op"] == "attend":
        more = dict(weight=s["weight"], weight_out=s["weight_out"], decay=0.998) if case["weight"] else {}
        if case["dtype"] == "int8":
            more["scale_out"] = s["scale_out"]
        if case["L"] > 1:
            more["n_new"] = s["n_new"]
        out = ia.cache_forward(_cache(s), s["q"], s["scale_q"], dtype=DTYPES[case["dtype"]], max_len=case["hi"], **more)
        return dict(out=out, weight=s["weight_out"]) if case["weight"] else dict(out=out)
    ia.cache_evict(_cache(s), case["keep"], s["weight"], order=s["order"], total=s["total"], sink=case["sink"], recent=case["recent"], max_len=case["hi"],
                   weight_out=s["weight_out"], order_out=s["order_out"], lens_out=s["lens_out"])
    return _evicted(s)


def _evicted(s):
    return dict(k_pages=s["k_pages"], v_pages=s["v_pages"], weight=s["weight_out"], order=s["order_out"], lens=s["lens_out"])


# ---------------------------------------------------------------- the plain forms


def _rotate(x, pos, freq, axis, rot, pairing, sign, wide):
    """x [B, H, L, d] turned pair by pair, in 64 bits or in 32; angles in 64.  The channels behind the first `rot` are kept."""
    angle = pos[axis].permute(1, 2, 0).double() * freq  # [B, L, rot / 2]
    t = torch.float64 if wide else torch.float32
    cos, sin = torch.cos(angle).to(t)[:, None], (sign * torch.sin(angle)).to(t)[:, None]
    y = x.to(t)
    if pairing == "adjacent":
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((turned, y[..., rot:]), dim=-1)


def _int8(x, scale):
    """rint(fl32(x / scale)) clamped; the quotient of two 32-bit numbers in 64 bits, rounded to 32, is their 32-bit quotient."""
    return torch.round((x.double() / scale.double()).float()).clamp_(-127, 127).to(torch.int8)


def _run_rope(s):
    case = s["case"]
    sign = -1.0 if case["inverse"] else 1.0
    q, k = (_rotate(x, s["pos"], s["freq"], s["axis_dev"], case["rot"], case["pairing"], sign, False).to(x.dtype) for x in (s["q"], s["k"]))
    return dict(q=q, k=k)


def _slots(s, index):
    """Page and place in it of the keys numbered index [B, n]."""
    page = s["case"]["page"]
    return torch.gather(s["table"].long(), 1, index // page), index % page


def _run_append(s):
    case = s["case"]
    q, k = s["q"].float(), s["k"].float()
    if case["rot"]:
        q, k = (_rotate(x, s["pos"], s["freq"], s["axis_dev"], case["rot"], case["pairing"], 1.0, True).float() for x in (q, k))
    scale_q = (q.abs().amax(dim=3).clamp(min=1e-12).double() / 127).float()
    token = torch.arange(case["L"], device="cuda")[None, :]
    there = token < s["n_new"][:, None]
    page, place = _slots(s, ((s["lens"] - s["n_new"])[:, None] + token).clamp(max=s["table"].shape[1] * case["page"] - 1))
    page, place = page[there], place[there]  # the tokens that are no padding
    for x, scale, pages in ((k, s["scale_k"], s["k_pages"]), (s["v"].float(), s["scale_v"], s["v_pages"])):
        pages[page, :, place] = _int8(x, scale[None, :, None, None]).transpose(1, 2)[there]
    there = there[:, None]
    return dict(q=_int8(q, scale_q[..., None]) * there[..., None], scale_q=torch.where(there, scale_q, torch.zeros_like(scale_q)), k_pages=s["k_pages"], v_pages=s["v_pages"])


def _run_attend(s):
    case = s["case"]
    B, Hq, L, d = s["q"].shape
    Hkv, hi = case["Hkv"], case["hi"]
    G = Hq // Hkv
    key = torch.arange(hi, device="cuda")
    page, place = _slots(s, key[None, :].expand(B, hi))
    k, v = (x[page, :, place].permute(0, 2, 1, 3) for x in (s["k_pages"], s["v_pages"]))  # [B, Hkv, hi, d]
    # sums of INT8 products stay below 2^24: exact in 32 bits
    a = torch.matmul(s["q"].float().reshape(B, Hkv, G * L, d), k.float().transpose(2, 3).contiguous()).to(torch.int32).reshape(B, Hkv, G, L, hi)
    token = torch.arange(L, device="cuda")[None, :, None]
    n_new = s["n_new"][:, None, None]
    sees = (token < n_new) & (key <= s["lens"][:, None, None] - n_new + token)  # [B, L, hi]
    sees = sees[:, None, None]
    lowest = -(1 << 30)
    a = torch.where(sees, a, torch.full_like(a, lowest))
    scale_q = s["scale_q"].double().reshape(B, Hkv, G, L)
    alpha = scale_q * s["scale_k"].double()[None, :, None, None] / math.sqrt(d)
    c = torch.floor(CLIP / alpha + 0.5).clamp(1, 1 << 30).long()[..., None]
    delta = torch.minimum((a.amax(dim=4, keepdim=True) - a).long(), c)
    index = torch.div(2 * TOP * delta + c, 2 * c, rounding_mode="floor")
    lut = torch.floor(255 * torch.exp(-CLIP * torch.arange(TOP + 1, device="cuda", dtype=torch.float64) / TOP) + 0.5).long()
    lut[TOP] = 0
    e = torch.where(sees, lut[index], torch.zeros_like(index))
    total = e.sum(dim=4, keepdim=True).clamp(min=1)
    p = torch.div(510 * e + total, 2 * total, rounding_mode="floor")
    acc = torch.matmul(p.float().reshape(B, Hkv, G * L, hi), v.float().contiguous()).reshape(B, Hkv, G, L, d)
    scale_v = s["scale_v"].double().reshape(1, -1, 1, 1, 1)
    if case["dtype"] == "int8":
        r = scale_v / (255 * s["scale_out"].double().reshape(1, -1, G if case["per_head"] else 1, 1, 1))
        m, power = torch.frexp(r)
        m = torch.floor(m * 2147483648.0 + 0.5).long()
        shift = 31 - power.long()
        out = ((acc.long() * m + (torch.ones_like(shift) << (shift - 1))) >> shift).clamp(-127, 127)
    else:
        out = acc * (scale_v / 255).float()
    got = dict(out=out.reshape(B, Hq, L, d).to(DTYPES[case["dtype"]]))
    if case["weight"]:
        drawn = (e.float() / total.float()).sum(dim=(2, 3))
        new = torch.where(key < s["lens"][:, None, None], 0.998 * s["weight"] + drawn, s["weight"])
        s["weight_out"].copy_(new)
        got["weight"] = s["weight_out"]
    return got


def _run_evict(s):
    case = s["case"]
    B, Hkv, hi, keep = case["B"], case["Hkv"], case["hi"], case["keep"]
    slot = torch.arange(hi, device="cuda")[None, None, :]
    n = s["lens"].long()[:, None, None]
    w = torch.where((s["order"] < case["sink"]) | (s["order"] >= s["total"][:, None, None] - case["recent"]), torch.full_like(s["weight"], math.inf), s["weight"])
    w = torch.where(slot < n, w, torch.full_like(w, -1.0))  # places behind the end come first, then the lightest, the oldest of equals
    by_order = torch.argsort(s["order"], dim=2, stable=True)
    rank = torch.argsort(torch.gather(w, 2, by_order), dim=2, stable=True)
    first = torch.gather(by_order, 2, rank)  # slots, the first to leave first
    place = torch.empty_like(first).scatter_(2, first, slot.expand(B, Hkv, hi).contiguous())
    gone = (place < hi - keep) & (slot < n) & (n > keep)
    stays = (slot < n) & ~gone
    hole, mover = gone & (slot < keep), stays & (slot >= keep) & (n > keep)
    b, h, to = hole.nonzero(as_tuple=True)  # the i-th hole of a head takes its i-th key from behind
    _, _, src = mover.nonzero(as_tuple=True)
    new, old = ((s["table"].long()[b, x // case["page"]], h, x % case["page"]) for x in (to, src))
    for pages in (s["k_pages"], s["v_pages"]):
        pages[new] = pages[old]
    under = slot < torch.minimum(n, torch.full_like(n, keep))
    for name in ("weight", "order"):
        x = s[name].clone()
        x[b, h, to] = s[name][b, h, src]
        s[name + "_out"].copy_(torch.where(under, x, s[name + "_out"]))
    s["lens_out"].copy_(s["lens"].clamp(max=keep))
    return _evicted(s)


def run(state):
    if own:
        return _run_own(state)
    return {"rope": _run_rope, "append": _run_append, "attend": _run_attend, "evict": _run_evict}[state["case"]["op"]](state)


def work(case):
    size = {"float32": 4, "float16": 2, "bfloat16": 2, "int8": 1}[case.get("dtype", "int8")]
    B, Hkv, d = case["B"], case["Hkv"], case["d"]
    if case["op"] == "rope":
        n = B * case["L"] * (case["Hq"] + Hkv) * d
        return {"bytes": 2 * n * size, "flops": 3 * n}
    keys = float(_lens(case).sum())
    if case["op"] == "append":
        new = float(_lens(case).clamp(max=case["L"]).sum())
        n = new * (case["Hq"] + 2 * Hkv) * d
        return {"bytes": n * (size + 1) + 4 * new * case["Hq"], "flops": 6 * n}
    if case["op"] == "attend":
        rows = B * case["Hq"] * case["L"]
        return {"bytes": keys * Hkv * (2 * d + (8 if case["weight"] else 0)) + rows * (d + 4 + d * size), "flops": 4.0 * keys * case["Hq"] * case["L"] * d}
    # weights and orders of every key; the keys moved: those behind the new end that stay, at most as many as leave
    lens = _lens(case).double()
    leave = (lens - case["keep"]).clamp(min=0)
    moved = float(torch.minimum(leave * case["keep"] / lens, torch.full_like(leave, case["keep"])).sum())
    return {"bytes": Hkv * (keys * 8 + moved * (4 * d + 8)), "flops": 4 * keys * Hkv}


# ---------------------------------------------------------------- the definition in 64 bits


def _host(x):
    return x.cpu().numpy()


def _exact_turn(x, pos, freq, axis, rot, pairing, inverse):
    """Each pair (a, b) as the complex number a + i b times exp(i angle)."""
    x = x.astype(np.float64)
    angle = np.moveaxis(pos.astype(np.float64)[axis], 0, 2) * freq[None, None, :]
    turn = np.exp((-1j if inverse else 1j) * angle)[:, None]
    lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if pairing == "adjacent" else (slice(0, rot // 2), slice(rot // 2, rot))
    z = (x[..., lo] + 1j * x[..., hi]) * turn
    y = x.copy()
    y[..., lo], y[..., hi] = z.real, z.imag
    return y


def _exact_evict(s):
    """One head after the other: sort, let the first of the order go, and fill the gaps from behind."""
    case = s["case"]
    lens, total, order, weight = (_host(s[name]) for name in ("lens", "total", "order", "weight"))
    new_order, new_weight, keep = order.copy(), weight.astype(np.float64), case["keep"]
    for b in range(case["B"]):
        n = int(lens[b])
        for h in range(case["Hkv"] if n > keep else 0):
            o, w = order[b, h, :n], weight[b, h, :n]
            held = (o < case["sink"]) | (o >= total[b] - case["recent"])
            leaves = np.zeros(n, dtype=bool)
            leaves[np.lexsort((o, w, held))[:n - keep]] = True
            gaps, behind = np.flatnonzero(leaves[:keep]), keep + np.flatnonzero(~leaves[keep:])
            new_order[b, h, gaps], new_weight[b, h, gaps] = o[behind], w[behind]
    return dict(k_pages=None, v_pages=None, weight=new_weight, order=new_order, lens=np.minimum(lens, keep))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        args = (_host(s["pos"]), _host(s["freq"]), s["axis"], case["rot"], case["pairing"], case["inverse"])
        return {name: _exact_turn(_host(s[name].float()), *args) for name in ("q", "k")}
    if case["op"] == "append":
        if work(case)["bytes"] > 2e8:
            return None
        x = _host(s["q"].float())
        if case["rot"]:
            x = _exact_turn(x, _host(s["pos"]), _host(s["freq"]), s["axis"], case["rot"], case["pairing"], False)
        scale = np.maximum(np.abs(x).max(axis=3), 1e-12) / 127
        token = np.arange(case["L"])[None, None, :]
        return dict(q=None, scale_q=np.where(token < _host(s["n_new"])[:, None, None], scale, 0.0), k_pages=None, v_pages=None)
    if case["op"] == "evict":
        return _exact_evict(s)
    if work(case)["flops"] > 2e10:
        return None
    B, Hq, L, d = s["q"].shape
    Hkv, n_all, page = case["Hkv"], _host(s["lens"]), case["page"]
    G = Hq // Hkv
    q, table, n_new = _host(s["q"]).astype(np.float64), _host(s["table"]), _host(s["n_new"])
    scale_q, scale_k, scale_v, scale_out = (_host(s[name]).astype(np.float64) for name in ("scale_q", "scale_k", "scale_v", "scale_out"))
    lut = np.array([math.floor(255 * math.exp(-CLIP * i / TOP) + 0.5) for i in range(TOP)] + [0], dtype=np.int64)
    out = np.zeros((B, Hq, L, d))
    weight = _host(s["weight"]).astype(np.float64) if case["weight"] else None
    for b in range(B):
        ids = torch.from_numpy(table[b, :-(-int(n_all[b]) // page)].astype(np.int64)).cuda()
        kb, vb = (_host(x[ids].transpose(1, 2).reshape(-1, Hkv, d)[:n_all[b]]) for x in (s["k_pages"], s["v_pages"]))
        for h in range(Hkv):
            kh, vh = kb[:, h].astype(np.float64), vb[:, h].astype(np.float64)
            if weight is not None:
                weight[b, h, :n_all[b]] *= 0.998
            for r in range(G * L):
                head, i = h * G + r // L, r % L
                if i >= n_new[b]:  # padding
                    continue
                n = int(n_all[b]) - int(n_new[b]) + i + 1
                logits = (kh[:n] @ q[b, head, i]).astype(np.int64)
                c = min(max(math.floor(CLIP * math.sqrt(d) / (scale_q[b, head, i] * scale_k[h if scale_k.size > 1 else 0]) + 0.5), 1), 1 << 30)
                away = np.minimum(logits.max() - logits, c)
                e = lut[(2 * TOP * away + c) // (2 * c)]
                p = (510 * e + e.sum()) // (2 * e.sum())
                acc, one_v = p.astype(np.float64) @ vh[:n], scale_v[h if scale_v.size > 1 else 0]
                if case["dtype"] == "int8":
                    m, power = math.frexp(one_v / (255 * float(scale_out[head if scale_out.size > 1 else 0])))
                    acc = acc.astype(np.int64) * math.floor(m * 2.0 ** 31 + 0.5)
                    out[b, head, i] = np.clip((acc + (1 << (30 - power))) >> (31 - power), -127, 127)
                else:
                    out[b, head, i] = acc * one_v / 255
                if weight is not None:
                    weight[b, h, :n] += e / e.sum()
    got = dict(out=out.astype(np.int8) if case["dtype"] == "int8" else out)
    return dict(got, weight=weight) if case["weight"] else got
