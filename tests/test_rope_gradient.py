"""IntAttn.rope under autograd: its gradient against the formula in 64 bits and against differences, gradients of any strides, several
graphs, a captured pass; and what is refused (on the CPU)."""
import numpy as np
import pytest

import cache_plain as plain
from test_cache_ops_gpu import dev, half_step, ia, rope_case, torch, wide  # noqa: F401 (fixtures)


# ---------------------------------------------------------------- refusals, which come before anything of a device is asked for

@pytest.fixture(scope="module")
def host():
    import os

    import torch  # noqa: F401 (before the library, which uses the HIP runtime that is loaded)

    from paper_2511_21513_amd import binding

    if not os.path.exists(binding.LIB_PATH):
        from paper_2511_21513_amd import build

        build.build()
    c = binding.IntAttn(device=-1)
    yield c
    c.close()


def test_outputs_that_autograd_would_not_see_are_refused(host):
    import torch

    x, pos, freq = torch.ones((1, 2, 3, 16)), torch.zeros((1, 1, 3), dtype=torch.int32), torch.ones(8, dtype=torch.float64)
    leaf = torch.ones((1, 2, 3, 16), requires_grad=True)
    for args, out in (((leaf, pos, freq), leaf), ((x, pos, freq), leaf), ((leaf, pos, freq), x), (([x, leaf], pos, freq), [x, x]), (([x, x], pos, freq), [x, leaf]),
                      ((leaf * 2, pos, freq), x)):
        with pytest.raises(ValueError, match="out does not go"):
            host.rope(*args, out=out)
    with pytest.raises(ValueError, match="freq has no gradient"):
        host.rope(x, pos, freq.clone().requires_grad_(True))
    with torch.no_grad():  # nothing to see: the checks that follow speak, of tensors that are not on the GPU
        with pytest.raises(Exception, match="not|device|CUDA|cuda|host-only"):
            host.rope(leaf, pos, freq, out=leaf)


# ---------------------------------------------------------------- gradients

CASES = [
    # dtype, B, L, heads, d, rot, axes, halves, far, inverse
    ("float32", 2, 5, (3, 1), 64, 64, 1, False, 100000, False),
    ("float32", 1, 9, (2,), 128, 32, 3, True, 5000, True),
    ("bfloat16", 3, 1, (8, 2), 128, 128, 1, False, 4000, False),
    ("float16", 1, 70, (4, 4), 64, 48, 2, True, 2000, False),
    ("float32", 1, 1, (1,), 16, 16, 4, False, 3, True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["heads first", "tokens first", "broadcast"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_gradient_is_the_formula_s(torch, ia, case, layout):
    dtype, B, L, heads, d, rot, axes, halves, far, inverse = case
    xs, pos, freq, axis = rope_case(len(str(case)), B, L, heads, d, rot, axes, far)
    leaves = [dev(torch, x, dtype).requires_grad_(True) for x in xs]
    rng = np.random.default_rng(1)
    gs = [dev(torch, rng.standard_normal(x.shape).astype(np.float32), dtype) for x in xs]
    order = list(axis)
    ys = ia.rope(leaves if len(leaves) > 1 else leaves[0], dev(torch, pos), dev(torch, freq), axis=order, pairing="halves" if halves else "adjacent", inverse=inverse)
    order.reverse()  # the call has its own copy
    ys = ys if len(leaves) > 1 else [ys]
    want_y = [plain.turned(wide(x.detach()), pos, freq, axis, halves, inverse) for x in leaves]
    if layout == "tokens first":
        gs = [g.transpose(1, 2).contiguous().transpose(1, 2) for g in gs]
    if layout == "broadcast":  # as a sum hands on: every stride 0
        gs = [torch.ones((), device="cuda", dtype=g.dtype).expand(g.shape) for g in gs]
    torch.autograd.backward(ys, gs)
    torch.cuda.synchronize()
    for x, y, g, w in zip(leaves, ys, gs, want_y):
        # roundings: to 32 bits, and to the type; the angle's product in 64 bits, by 2^-53 of up to far radians, turns by as much
        for got, want, size in ((y.detach(), w, np.abs(wide(x.detach())).max()),
                                (x.grad, plain.turned(wide(g), pos, freq, axis, halves, not inverse), np.abs(wide(g)).max())):
            limit = (half_step(torch, dtype) * 1.0001 + (2.0 ** -24 if dtype != "float32" else 0)) * np.abs(want) + size * (far * 2.0 ** -51 + 2.0 ** -50) + (2.0 ** -25 if dtype == "float16" else 0)
            assert got.dtype is x.dtype and (np.abs(wide(got) - want) <= limit).all()


@pytest.mark.gpu
def test_gradient_against_differences(torch, ia):
    """The slope of sum(g rope(x)) in twenty directions; the map is linear, so a difference has no error but roundings."""
    xs, pos, freq, axis = rope_case(3, 2, 19, (3,), 64, 64, 3, 50)
    rng = np.random.default_rng(5)
    g = rng.standard_normal(xs[0].shape).astype(np.float32)
    x = dev(torch, xs[0]).requires_grad_(True)
    (ia.rope(x, dev(torch, pos), dev(torch, freq), axis=axis) * dev(torch, g)).sum().backward()
    grad = wide(x.grad)
    for _ in range(20):
        way = rng.integers(-2, 3, xs[0].shape).astype(np.float64)
        slope = ((plain.turned(xs[0] + way, pos, freq, axis, False) - plain.turned(xs[0] - way, pos, freq, axis, False)) * g).sum() / 2
        size = (np.abs(grad) * np.abs(way)).sum()
        assert abs((grad * way).sum() - slope) <= 2.0 ** -24 * size + 1e-9 * size


@pytest.mark.gpu
def test_gradients_that_arrive_in_other_places(torch, ia):
    """Gradients that start off 16 bytes, an output that nothing uses, one input that needs none, and a gradient of the gradient."""
    xs, pos, freq, axis = rope_case(4, 2, 6, (3, 2), 64, 64, 2, 300)
    pos, freq = dev(torch, pos), dev(torch, freq)
    turn = lambda t, inverse=False: ia.rope(t, pos, freq, axis=axis, inverse=inverse)
    q, k = (dev(torch, x).requires_grad_(True) for x in xs)
    flat = torch.randn(q.numel() + 1, device="cuda")
    off = flat[1:].view(q.shape)  # 4 bytes off
    assert off.data_ptr() % 16 == 4
    grad, = torch.autograd.grad(turn(q), q, off)
    assert torch.equal(grad, turn(off.clone(), True))
    wide_rows = torch.randn(q.shape[:3] + (65,), device="cuda")[..., :64]  # rows 260 bytes apart
    grad, = torch.autograd.grad(turn(q), q, wide_rows)
    assert torch.equal(grad, turn(wide_rows.contiguous(), True))
    a, b = turn([q, k])
    g = torch.randn_like(b)
    none, grad = torch.autograd.grad(b, (q, k), g, allow_unused=True)
    assert none is None and torch.equal(grad, turn(g, True))
    a, b = turn([q.detach(), k])
    assert not a.requires_grad and b.requires_grad
    grad, = torch.autograd.grad(b, k, g)
    assert torch.equal(grad, turn(g, True))
    # of the gradient: rope again
    g = torch.randn_like(q).requires_grad_(True)
    first, = torch.autograd.grad(turn(q), q, g, create_graph=True)
    h = torch.randn_like(q)
    second, = torch.autograd.grad(first, g, h)
    assert torch.equal(second, turn(h))
    with torch.no_grad():
        assert not turn(q).requires_grad


@pytest.mark.gpu
def test_tensors_changed_in_place_are_noticed(torch, ia):
    xs, pos, freq, axis = rope_case(5, 1, 6, (3,), 64, 64, 1, 300)
    p, f = dev(torch, pos), dev(torch, freq)
    x = dev(torch, xs[0]).requires_grad_(True)
    y = ia.rope(x, p, f)
    p += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    w, z = torch.ones(64, device="cuda", requires_grad=True), dev(torch, xs[0])
    y = w * z  # keeps z for w's gradient
    ia.rope(z, p, f, out=z)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


@pytest.mark.gpu
def test_training_step_in_a_graph(torch, ia):
    """Forward and backward captured together; every replay against the eager step on the same values."""
    xs, pos, freq, axis = rope_case(6, 2, 33, (4, 2), 64, 64, 1, 3000)
    p, f = dev(torch, pos), dev(torch, freq)
    q, k = (dev(torch, x) for x in xs)
    wq, wk = (torch.randn_like(t) for t in (q, k))

    def step(q, k):
        q, k = q.detach().requires_grad_(True), k.detach().requires_grad_(True)
        a, b = ia.rope([q, k], p, f)
        return (a, b) + torch.autograd.grad((a, b), (q, k), (wq, wk))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(q, k)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        got = step(q, k)
    for _ in range(3):
        for t in (q, k, wq, wk):
            t.copy_(torch.randn_like(t))
        p.copy_(torch.randint_like(p, 0, 9000))
        graph.replay()
        torch.cuda.synchronize()
        want = step(q, k)
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y)
