"""Argument checks of the operators around the paged cache, on a host-only context: a call that passes them is refused for want of a
device, any other names what is wrong with it.  No GPU; the struct layouts are compared with the header's."""
import ctypes
import os
import subprocess

import pytest

from paper_2511_21513_amd import binding

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "intattn.h")
P = 1 << 20  # an address that is aligned and never followed


@pytest.fixture(scope="module")
def ia():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2511_21513_amd import build

        build.build()
    c = binding.IntAttn(device=-1)
    yield c
    c.close()


def cache(**kw):
    c = binding.Cache()
    c.B, c.Hkv, c.d, c.n_pages, c.page_size, c.max_pages = 2, 4, 64, 10, 16, 5
    c.k, c.v, c.table, c.lens, c.scale_k, c.scale_v = P, P, P, P, P, P
    c.k_stride[:] = c.v_stride[:] = (4 * 16 * 64, 16 * 64, 64)
    c.table_stride = 5
    return put(c, kw)


def put(a, kw):
    for name, value in kw.items():
        field = getattr(a, name)
        if isinstance(value, tuple):
            i, value = value
            field[i] = value
        else:
            setattr(a, name, value)
    return a


def rotary(r, **kw):
    r.rot, r.n_axes, r.pos, r.freq = 64, 1, P, P
    return put(r, kw)


def rope(rot=None, **kw):
    a = binding.RopeArgs()
    a.B, a.L, a.d, a.dtype = 2, 3, 64, 2
    a.H[0], a.H[1] = 8, 2
    for i in range(2):
        a.src[i], a.dst[i] = P, P + (1 << 24)
        a.src_stride[i][:] = a.dst_stride[i][:] = (8 * 3 * 128, 3 * 128, 128)
    rotary(a.rotary, **(rot or {}))
    return put(a, kw)


def append(rot=None, **kw):
    a = binding.AppendArgs()
    a.L, a.Hq, a.dtype = 3, 8, 1
    a.q, a.k, a.v, a.q_out, a.q_scale = P, P, P, P, P
    a.q_stride[:] = a.k_stride[:] = a.v_stride[:] = (3 * 8 * 128, 128, 8 * 128)
    a.q_out_stride[:] = (3 * 8 * 64, 3 * 64, 64)
    rotary(a.rotary, **(rot or {}))
    return put(a, kw)


def forward(**kw):
    a = binding.CacheForwardArgs()
    a.Hq, a.L, a.out_type = 8, 2, 2
    a.q, a.scale_q, a.out = P, P, P
    a.q_stride[:] = (8 * 2 * 64, 2 * 64, 64)
    a.out_stride[:] = (8 * 2 * 128, 2 * 128, 128)
    a.weight, a.weight_out, a.decay = P, P, 1.0
    a.weight_stride[:] = a.weight_out_stride[:] = (320, 80)
    return put(a, kw)


def evict(**kw):
    a = binding.EvictArgs()
    a.keep = 20
    a.weight, a.weight_out, a.order, a.order_out, a.lens_out = P, P, P, P, P
    for s in (a.weight_stride, a.weight_out_stride, a.order_stride, a.order_out_stride):
        s[:] = (320, 80)
    return put(a, kw)


def code(ia, name, *args):
    rc = getattr(ia._lib, name)(ia._ctx, *(ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args))
    return rc, ia.last_error()


CALLS = {"intattn_cache_append": append, "intattn_cache_forward": forward, "intattn_cache_evict": evict}
BAD, NOT = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED


def test_calls_that_pass_the_checks_want_a_device(ia):
    for name, make in CALLS.items():
        rc, text = code(ia, name, cache(), make(), None)
        assert rc == NOT and "host-only" in text, (name, rc, text)
    rc, text = code(ia, "intattn_rope", rope(), None)
    assert rc == NOT and "host-only" in text
    rc, text = code(ia, "intattn_cache_reserve", cache(), 16, 5, 0)
    assert rc == NOT and "host-only" in text


def test_null_arguments(ia):
    for name, make in CALLS.items():
        fn = getattr(ia._lib, name)
        assert fn(ia._ctx, ctypes.byref(cache()), None, None) == BAD
        assert fn(ia._ctx, None, ctypes.byref(make()), None) == BAD
        assert fn(None, ctypes.byref(cache()), ctypes.byref(make()), None) == BAD
    assert ia._lib.intattn_rope(ia._ctx, None, None) == BAD
    assert ia._lib.intattn_rope(None, ctypes.byref(rope()), None) == BAD
    assert ia._lib.intattn_cache_reserve(ia._ctx, None, 1, 1, 0) == BAD


@pytest.mark.parametrize("want, kw", [
    (BAD, dict(B=0)), (BAD, dict(Hkv=0)), (BAD, dict(n_pages=0)), (BAD, dict(page_size=0)), (BAD, dict(max_pages=0)), (NOT, dict(d=96)),
    (NOT, dict(B=65536)), (NOT, dict(B=30000, table_stride=5)), (NOT, dict(page_size=65537)), (NOT, dict(max_pages=1 << 27)),
    (BAD, dict(scale_mode=2)), (BAD, dict(scale_mode=-1)), (BAD, dict(reserved=1)), (BAD, dict(k=None)), (BAD, dict(v=None)), (BAD, dict(table=None)),
    (BAD, dict(lens=None)), (BAD, dict(scale_k=None)), (BAD, dict(scale_v=None)), (BAD, dict(k=P + 8)), (BAD, dict(v=P + 8)), (BAD, dict(k_stride=(0, 24))),
    (BAD, dict(v_stride=(1, -16))), (BAD, dict(k_stride=(2, 48))), (BAD, dict(table=P + 2)), (BAD, dict(lens=P + 1)), (BAD, dict(scale_k=P + 2)), (BAD, dict(table_stride=4)),
])
def test_caches_that_are_refused(ia, want, kw):
    for name, make in CALLS.items():
        rc, text = code(ia, name, cache(**kw), make(Hq=max(8, 8 * (kw.get("B", 1) > 9))) if name != "intattn_cache_evict" else make(), None)
        assert rc == want and text and "host-only" not in text, (name, kw, rc, text)
    assert code(ia, "intattn_cache_reserve", cache(**kw), 1, 1, 0)[0] == want


@pytest.mark.parametrize("want, kw", [
    (BAD, dict(Hq=0)), (BAD, dict(L=0)), (BAD, dict(Hq=6)), (NOT, dict(L=2049)), (BAD, dict(max_len=-1)), (BAD, dict(out_type=4)), (BAD, dict(out_type=-1)),
    (BAD, dict(scale_out_mode=2)), (BAD, dict(scale_out_mode=-1)), (BAD, dict(q=None)), (BAD, dict(scale_q=None)), (BAD, dict(out=None)), (BAD, dict(q=P + 8)), (BAD, dict(out=P + 4)), (BAD, dict(q_stride=(1, 40))),
    (BAD, dict(out_stride=(2, 72))), (BAD, dict(scale_q=P + 2)), (BAD, dict(n_new=P + 1)), (BAD, dict(weight=None)), (BAD, dict(weight_out=None)), (BAD, dict(weight_stride=(0, -4))),
    (BAD, dict(weight_out_stride=(1, 81))), (BAD, dict(decay=float("nan"))), (BAD, dict(decay=float("inf"))),
])
def test_forwards_that_are_refused(ia, want, kw):
    rc, text = code(ia, "intattn_cache_forward", cache(), forward(**kw), None)
    assert rc == want and text and "host-only" not in text, (rc, text)


def test_long_sequences_need_a_bound(ia):
    long = cache(max_pages=8193, table_stride=8193)
    for name, make in (("intattn_cache_forward", forward), ("intattn_cache_evict", evict)):
        rc, text = code(ia, name, long, make(), None)
        assert rc == NOT and "131071" in text
        assert "host-only" in code(ia, name, long, make(max_len=131071), None)[1]
        assert code(ia, name, long, make(max_len=131072), None)[0] == NOT


@pytest.mark.parametrize("want, kw", [
    (BAD, dict(L=0)), (NOT, dict(L=131072)), (BAD, dict(Hq=-4)), (BAD, dict(Hq=6)), (NOT, dict(Hq=2044)), (BAD, dict(dtype=3)), (BAD, dict(dtype=-1)), (BAD, dict(reserved=1)),
    (BAD, dict(k=None)), (BAD, dict(v=None)), (BAD, dict(q=None)), (BAD, dict(q_out=None)), (BAD, dict(q_scale=None)), (BAD, dict(rot=dict(inverse=1))), (BAD, dict(k=P + 8)),
    (BAD, dict(v_stride=(2, 24))), (BAD, dict(q_out_stride=(1, 72))), (BAD, dict(q_scale=P + 2)), (BAD, dict(n_new=P + 1)), (BAD, dict(order=P + 2)), (BAD, dict(weight=P, weight_stride=(0, -1))),
])
def test_appends_that_are_refused(ia, want, kw):
    rc, text = code(ia, "intattn_cache_append", cache(), append(**kw), None)
    assert rc == want and text and "host-only" not in text, (rc, text)


def test_outputs_over_themselves_are_refused(ia):
    """Inputs may have axes of stride 0, what is written may not; an axis of one element may have any stride."""
    for i, s in ((0, 0), (0, 1), (1, 1), (0, 2)):
        a = rope()
        a.dst_stride[i][s] = 112
        assert code(ia, "intattn_rope", a, None)[0] == BAD
        a = rope()
        a.src_stride[i][s] = 0
        assert "host-only" in code(ia, "intattn_rope", a, None)[1]
    for s in range(3):
        assert code(ia, "intattn_cache_append", cache(), append(q_out_stride=(s, 48)), None)[0] == BAD
        assert "host-only" in code(ia, "intattn_cache_append", cache(), append(q_stride=(s, 0)), None)[1]
        assert code(ia, "intattn_cache_forward", cache(), forward(out_stride=(s, 48)), None)[0] == BAD
        assert "host-only" in code(ia, "intattn_cache_forward", cache(), forward(q_stride=(s, 0)), None)[1]
    for s in range(2):
        for name in ("k_stride", "v_stride"):
            flat = cache(**{name: (s, 0)})
            assert code(ia, "intattn_cache_append", flat, append(), None)[0] == BAD
            assert code(ia, "intattn_cache_evict", flat, evict(), None)[0] == BAD
            assert "host-only" in code(ia, "intattn_cache_forward", flat, forward(), None)[1]
        assert code(ia, "intattn_cache_append", cache(), append(weight=P, weight_stride=(s, 0)), None)[0] == BAD
        assert code(ia, "intattn_cache_append", cache(), append(order=P, order_stride=(s, 0)), None)[0] == BAD
        assert code(ia, "intattn_cache_forward", cache(), forward(weight=P, weight_out=P + 4096, weight_out_stride=(s, 0)), None)[0] == BAD
        assert "host-only" in code(ia, "intattn_cache_forward", cache(), forward(weight=P, weight_out=P + 4096, weight_stride=(s, 0)), None)[1]
        assert code(ia, "intattn_cache_evict", cache(), evict(weight_out=P + 4096, weight_out_stride=(s, 0)), None)[0] == BAD
        assert code(ia, "intattn_cache_evict", cache(), evict(order=P, order_out=P + 4096, order_out_stride=(s, 0)), None)[0] == BAD
    assert "host-only" in code(ia, "intattn_rope", one_token(), None)[1]


def one_token():
    a = rope(B=1, L=1)
    for i in range(2):
        a.dst_stride[i][0] = a.dst_stride[i][2] = 0
    return a


def test_calls_of_more_tokens_than_a_grid_has_workgroups(ia):
    """2^24 workgroups of 256 threads are 2^32 threads."""
    for B, L, want in ((4096, 4096, NOT), (4095, 4096, None), (1, 131071, None), (65535, 256, None), (65535, 257, NOT)):
        a = append(L=L)
        rc, text = code(ia, "intattn_cache_append", cache(B=B, Hkv=1), a, None)
        assert (rc == want and "2^24" in text) if want else "host-only" in text, (B, L, rc, text)
    for L, want in ((1 << 23, NOT), ((1 << 23) - 1, None)):
        rc, text = code(ia, "intattn_rope", rope(L=L), None)
        assert (rc == want and "2^24" in text) if want else "host-only" in text, (L, rc, text)


def test_appends_without_queries_or_rotation_pass(ia):
    rc, text = code(ia, "intattn_cache_append", cache(), append(Hq=0, q=None, q_out=None, q_scale=None, rot=dict(rot=0, pos=None, freq=None)), None)
    assert "host-only" in text


@pytest.mark.parametrize("want, kw", [
    (NOT, dict(rot=8)), (NOT, dict(rot=24)), (NOT, dict(rot=80)), (NOT, dict(rot=-16)), (BAD, dict(pairing=2)), (BAD, dict(n_axes=0)), (BAD, dict(n_axes=5)), (BAD, dict(pos=None)),
    (BAD, dict(freq=None)), (BAD, dict(pos=P + 2)), (BAD, dict(freq=P + 4)), (BAD, dict(pos_stride=(0, -1))), (BAD, dict(axis=(31, 1))), (BAD, dict(n_axes=3, axis=(0, 3))),
])
def test_rotations_that_are_refused(ia, want, kw):
    for rc, text in (code(ia, "intattn_rope", rope(rot=kw), None), code(ia, "intattn_cache_append", cache(), append(rot=kw), None)):
        assert rc == want and text and "host-only" not in text, (kw, rc, text)
    assert code(ia, "intattn_rope", rope(rot=dict(inverse=2)), None)[0] == BAD
    assert code(ia, "intattn_rope", rope(rot=dict(rot=0)), None)[0] == NOT


@pytest.mark.parametrize("want, kw", [
    (BAD, dict(B=0)), (BAD, dict(L=0)), (BAD, dict(H=(0, 0))), (BAD, dict(H=(1, -1))), (NOT, dict(d=72)), (NOT, dict(d=2048)), (BAD, dict(dtype=3)), (NOT, dict(H=(0, 65535))),
    (NOT, dict(B=1 << 30)), (BAD, dict(src=(0, None))), (BAD, dict(dst=(1, None))), (BAD, dict(src=(1, P + 8))), (BAD, dict(dst=(0, P + 4))),
])
def test_ropes_that_are_refused(ia, want, kw):
    rc, text = code(ia, "intattn_rope", rope(**kw), None)
    assert rc == want and text and "host-only" not in text, (rc, text)


def test_rope_strides(ia):
    for field, i, s, value in (("src_stride", 0, 2, 120), ("dst_stride", 1, 0, -16), ("dst_stride", 0, 2, 112)):
        a = rope()
        getattr(a, field)[i][s] = value
        assert code(ia, "intattn_rope", a, None)[0] == BAD
    a = rope(dst=(0, P))  # in place
    assert "host-only" in code(ia, "intattn_rope", a, None)[1]
    a.dst_stride[0][1] += 16
    assert code(ia, "intattn_rope", a, None)[0] == BAD


@pytest.mark.parametrize("want, kw", [
    (BAD, dict(keep=0)), (BAD, dict(sink=-1)), (BAD, dict(recent=-1)), (BAD, dict(max_len=-2)), (BAD, dict(weight=None)), (BAD, dict(weight_out=None)), (BAD, dict(lens_out=None)),
    (BAD, dict(order=None)), (BAD, dict(order_out=None)), (BAD, dict(weight=P + 2)), (BAD, dict(total=P + 1)), (BAD, dict(weight_stride=(0, -1))), (BAD, dict(order_out_stride=(1, 82))),
])
def test_evictions_that_are_refused(ia, want, kw):
    rc, text = code(ia, "intattn_cache_evict", cache(), evict(**kw), None)
    assert rc == want and text and "host-only" not in text, (rc, text)


def test_reservations_that_are_refused(ia):
    assert code(ia, "intattn_cache_reserve", cache(), -1, 0, 0)[0] == BAD
    assert code(ia, "intattn_cache_reserve", cache(), 4097, 0, 0)[0] == BAD
    assert code(ia, "intattn_cache_reserve", cache(), 1, -1, 0)[0] == BAD
    assert code(ia, "intattn_cache_reserve", cache(), 1, 1, -1)[0] == BAD


def test_struct_layouts_match_the_header(tmp_path):
    structs = {"intattn_cache": binding.Cache, "intattn_rotary": binding.Rotary, "intattn_rope_args": binding.RopeArgs, "intattn_append_args": binding.AppendArgs,
               "intattn_cache_forward_args": binding.CacheForwardArgs, "intattn_evict_args": binding.EvictArgs}
    src, want = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{HEADER}"', "int main(void){"], []
    for name, s in structs.items():
        src.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(ctypes.sizeof(s))
        for f in s._fields_:
            src.append(f'printf("%zu\\n", offsetof({name}, {f[0]}));')
            want.append(getattr(s, f[0]).offset)
    (tmp_path / "probe.c").write_text("\n".join(src + ["return 0;}"]))
    subprocess.run(["gcc", "-std=c11", "-o", str(tmp_path / "probe"), str(tmp_path / "probe.c")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "probe")], check=True, capture_output=True, text=True).stdout.split()]
    assert got == want
