"""Room for scores of attention over the paged cache is bounded: calls with more take their KV heads one part after the other.  Parts of a
call are compared with calls on a few sequences each, whose room is below the bound."""
import numpy as np
import pytest

import cache_plain as plain
from test_cache_ops_gpu import Case, dev, torch, wide  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

GIB = 1 << 30


@pytest.fixture
def own(torch):
    from paper_2511_21513_amd import binding

    c = binding.IntAttn(device=0)
    yield c
    torch.cuda.synchronize()
    c.close()


def shared_pages(torch, B, Hkv, d, page, lens, seed):
    """Many sequences over the pages of a few: a large call on little memory."""
    from paper_2511_21513_amd import binding

    rng = np.random.default_rng(seed)
    width = -(-max(lens) // page)
    n_pages = 3 * width
    k, v = (dev(torch, rng.integers(-127, 128, (n_pages, Hkv, page, d)).astype(np.int8)) for _ in range(2))
    table = dev(torch, np.stack([rng.permutation(n_pages)[:width] for _ in range(B)]).astype(np.int32))
    n = dev(torch, np.array([lens[b % len(lens)] for b in range(B)], dtype=np.int32))
    sk, sv = (dev(torch, rng.uniform(0.005, 0.03, Hkv).astype(np.float32)) for _ in range(2))
    return lambda some: binding.PagedCache(k, v, table[some], n[some], sk, sv)


def used(torch, call):
    """Bytes of the GPU's memory that a call leaves allocated, outside torch's own."""
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    call()
    torch.cuda.synchronize()
    return free - torch.cuda.mem_get_info()[0]


@pytest.mark.parametrize("B, Hkv, L, lens", [
    (13, 3, 512, [8400, 7000, 500]),      # 1024 rows of 8400 keys: keys split, 34 MB of scores a KV head, 39 of them
    (700, 2, 512, [4500, 1000, 0, 17]),   # 1024 rows of up to 4500 keys: one launch for a part, 1.2 MB of weights a KV head, 1400 of them
], ids=str)
@pytest.mark.parametrize("weight", [False, True])
def test_parts_of_a_call_are_the_call(torch, own, B, Hkv, L, lens, weight):
    cache = shared_pages(torch, B, Hkv, 64, 64, lens, B)
    q = torch.randint(-127, 128, (B, 2 * Hkv, L, 64), device="cuda").to(torch.int8)
    s = torch.rand((B, 2 * Hkv, L), device="cuda") * 0.01 + 0.002
    w = torch.rand((B, Hkv, -(-max(lens) // 64) * 64), device="cuda") if weight else None
    out, w_out = torch.full_like(q, 99), None if w is None else torch.full_like(w, -3)
    whole = cache(slice(None))
    # (a process's first launches load code and take memory for themselves: those are another context's, on a part of the call)
    from paper_2511_21513_amd import binding

    other, few = binding.IntAttn(device=0), slice(0, max(1, B // 8))
    other.cache_forward(cache(few), q[few], s[few], dtype=torch.int8, weight=None if w is None else w[few], weight_out=None if w is None else w_out[few], decay=0.5)
    torch.cuda.synchronize()
    other.close()
    assert used(torch, lambda: own.cache_forward(whole, q, s, out=out, weight=w, weight_out=w_out, decay=0.5)) <= GIB + (64 << 20)
    for b in list(range(0, B, max(1, B // 7))) + [B - 1]:
        some = slice(b, b + 1)
        sw = None if w is None else torch.full_like(w[some], -3)
        got = own.cache_forward(cache(some), q[some], s[some], dtype=torch.int8, weight=None if w is None else w[some], weight_out=sw, decay=0.5)
        assert torch.equal(got, out[some])
        if weight:  # each of the 2 L rows adds a rounding, on either side
            n = lens[b % len(lens)]
            assert ((sw - w_out[some])[..., :n].abs() <= 2 * (2 * L + 3) * 2.0 ** -24 * w_out[some][..., :n]).all()
            assert (w_out[some][..., n:] == -3).all()


def test_the_largest_rooms_are_bounded(torch, own):
    """A reservation for 4096 rows of 64 KV heads over 32768 keys, which once was 34 GB, and then a captured call of that size."""
    B, Hkv, L, n = 8, 8, 4096, 32768
    cache = shared_pages(torch, B, Hkv, 64, 64, [n], 3)(slice(None))
    assert used(torch, lambda: own.cache_reserve(cache, rows=4096)) <= GIB + (64 << 20)
    q = torch.randint(-127, 128, (B, Hkv, L, 64), device="cuda").to(torch.int8)
    s = torch.rand((B, Hkv, L), device="cuda") * 0.01 + 0.002
    new = torch.ones(B, dtype=torch.int32, device="cuda")  # (one token each; the others are padding, which takes the same room)
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        own.cache_forward(cache, q, s, out=out, n_new=new)
    want = own.cache_forward(cache, q[:, :, :1].contiguous(), s[:, :, :1].contiguous(), dtype=torch.int8)
    for _ in range(2):
        out.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:, :, :1], want) and int((out[:, :, 1:] != 0).sum()) == 0


def test_room_does_not_double_past_the_bound(torch, own):
    """0.98 GB, and then a little more, up to the bound."""
    first, second = (shared_pages(torch, 64, 8, 64, 64, [n], 5)(slice(None)) for n in (30000, 31000))

    def grow():
        own.cache_reserve(first, rows=16)
        own.cache_reserve(second, rows=16)

    assert used(torch, grow) <= 2 * GIB + (64 << 20)


def test_parts_against_the_plain_form(torch, own):
    """One KV head to a part, each of more room than the bound alone, checked where the tokens are no padding."""
    c = Case(torch, 5, 2, 1, 64, 64, [66000, 65999], room=0)
    L, rng = 4096, np.random.default_rng(6)
    q = rng.integers(-127, 128, (2, 1, L, 64)).astype(np.int8)
    s = rng.uniform(0.002, 0.02, (2, 1, L)).astype(np.float32)
    new = np.array([2, 3], dtype=np.int32)
    w = rng.random((2, 1, c.width * 64)).astype(np.float32)
    wt = dev(torch, w)
    got = own.cache_forward(c.cache, dev(torch, q), dev(torch, s), dtype=torch.int8, n_new=dev(torch, new), weight=wt, decay=0.25)
    torch.cuda.synchronize()
    _, want, _, after = plain.attend(q, s, c.k, c.v, c.table, c.lens, c.sk, c.sv, n_new=new, weight=w, decay=0.25)
    assert int((got.cpu().numpy() != want).sum()) == 0
    assert (np.abs(wide(wt) - after) <= (3 + 3) * 2.0 ** -24 * after).all()  # (rows of padding add zeros)
