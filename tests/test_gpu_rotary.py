"""GPU: rotary positions of several axes (include/wht_rotary.h) against the definition in 64 bits, and their gradient against the formula's and
against differences."""
import math

import pytest
import torch

import attention4_check as check
import paper_2603_08343_amd as wht
from attention_check import HALF, same
from paper_2603_08343_amd import attention4
from paper_2603_08343_amd.autograd import WhtRotaryFunction, wht_rotary

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B16, F32 = torch.bfloat16, torch.float32

CASES = [  # T, heads, head_dim, rotary, sections, cyclic, interleaved, dtype
    (1, 1, 16, 16, (8,), False, False, B16),
    (1, 40, 128, 128, (16, 24, 24), False, False, B16),
    (7, 5, 64, 32, (4, 12), False, True, F32),
    (63, 12, 96, 96, (12, 18, 18), True, False, B16),
    (130, 3, 256, 256, (128,), False, False, F32),
    (65, 33, 48, 16, (2, 2, 2, 2), True, True, B16),
    (300, 2, 112, 64, (11, 21), False, False, F32),
    (257, 17, 80, 80, (40, 0), False, True, F32),
    (5, 1024, 16, 16, (3, 5), False, False, B16),
]


def make(T, heads, head_dim, rotary, sections, dtype, rows=40, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, heads, head_dim, generator=g).to(dtype).to(DEV)
    positions = torch.randint(0, rows, (T, len(sections)), generator=g).to(torch.int32).to(DEV)
    return x, positions, wht.wht_attention_rope_table(rows, rotary, device=DEV)


def want(x, rope, positions, axes, interleaved, back=False):
    y, size = check.turn(x, rope, positions.cpu().long()[:, list(axes)], interleaved, back)
    return y, size + HALF[x.dtype] * y.abs() * 1.01 + 1e-38


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_rotate(case, inverse):
    T, heads, head_dim, rotary, sections, cyclic, interleaved, dtype = case
    x, positions, rope = make(T, heads, head_dim, rotary, sections, dtype)
    axes = wht.wht_rotary_axes(sections, cyclic)
    y, tol = want(x, rope, positions, axes, interleaved, inverse)
    got = wht.wht_rotary_rotate(x, rope, positions, axes, interleaved, inverse)
    same(got, y, tol)
    back = x.clone()
    assert wht.wht_rotary_rotate(back, rope, positions, axes, interleaved, inverse, out=back) is back
    assert torch.equal(back, got)


def test_one_axis_and_the_rows_own_number():
    x, positions, rope = make(30, 4, 64, 64, (32,), B16)
    flat = wht.wht_rotary_rotate(x, rope, positions[:, 0].contiguous())
    assert torch.equal(flat, wht.wht_rotary_rotate(x, rope, positions))
    rows = torch.arange(30, dtype=torch.int32, device=DEV)
    assert torch.equal(wht.wht_rotary_rotate(x, rope), wht.wht_rotary_rotate(x, rope, rows))
    assert torch.equal(wht.wht_rotary_rotate(x, rope, axes=list(bytes(32))), wht.wht_rotary_rotate(x, rope))


def test_positions_outside_the_table_give_nan():
    x, positions, rope = make(6, 3, 64, 32, (8, 8, 0), B16)
    positions[1, 0], positions[2, 1], positions[3, 2], positions[4, 1] = 40, -1, 77, -2 ** 31          # an axis without a pair is not asked for
    axes = wht.wht_rotary_axes((8, 8, 0))
    y, tol = want(x, rope, positions, axes, False)
    same(wht.wht_rotary_rotate(x, rope, positions, axes), y, tol)


def test_append4_and_rotate_agree():
    """What the append does with queries is this, without the transform."""
    c = check.make4(2, [5, 8], [5, 8], (4, 2, 64), 16)
    positions = torch.randint(0, 40, (13, 3), dtype=torch.int32, device=DEV)
    rope, axes = wht.wht_attention_rope_table(40, 64, device=DEV), wht.wht_rotary_axes((8, 12, 12))
    q = wht.wht_attention_append4(c["q"], c["k"], c["v"], *(c[n] for n in ("k_pages", "v_pages", "k_scales", "v_scales")), c["table"], c["lengths"], rope,
                                  q_starts=c["starts"], positions=positions, axes=axes, transform=False)
    r = wht.wht_rotary_rotate(c["q"], rope, positions, axes)
    y, tol = want(c["q"], rope, positions, axes, False)
    same(q, y, tol)
    same(r, y, tol)


def test_strides_and_other_streams():
    fused = torch.randn(50, 10, 64, device=DEV).to(B16)
    x = fused[:, 1:7]
    _, positions, rope = make(50, 1, 64, 64, (16, 16), B16)
    axes = wht.wht_rotary_axes((16, 16))
    y = wht.wht_rotary_rotate(x.contiguous(), rope, positions, axes)
    assert torch.equal(wht.wht_rotary_rotate(x, rope, positions, axes), y)
    turned = x.transpose(0, 1).contiguous().transpose(0, 1)          # heads outside
    assert torch.equal(wht.wht_rotary_rotate(turned, rope, positions, axes), y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = wht.wht_rotary_rotate(x, rope, positions, axes, stream=side)
    side.synchronize()
    assert torch.equal(got, y)


@pytest.mark.parametrize("dtype", [B16, F32], ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_is_the_formulas(dtype, interleaved):
    x, positions, rope = make(70, 5, 96, 64, (10, 11, 11), dtype)
    axes = wht.wht_rotary_axes((10, 11, 11))
    dy = torch.randn(70, 5, 96, generator=torch.Generator().manual_seed(5)).to(dtype).to(DEV)
    x.requires_grad_(True)
    y = wht_rotary(x, rope, positions, axes, interleaved)
    forward, tol = want(x, rope, positions, axes, interleaved)
    same(y, forward, tol)
    dx, = torch.autograd.grad(y, x, dy)
    back, tol = want(dy, rope, positions, axes, interleaved, back=True)
    same(dx, back, tol)


def test_gradient_is_that_of_differences():
    """The operator is linear: a difference of outputs is a derivative up to the outputs' roundings, whatever its step."""
    x, positions, rope = make(4, 2, 32, 32, (8, 8), F32)
    axes = wht.wht_rotary_axes((8, 8))
    w = torch.randn(4, 2, 32, device=DEV)
    x.requires_grad_(True)
    (wht_rotary(x, rope, positions, axes) * w).sum().backward()
    for at in ((0, 0, 0), (1, 1, 17), (3, 0, 31), (2, 1, 8)):
        step = torch.zeros_like(x)
        step[at] = 0.5
        up, down = (wht.wht_rotary_rotate((x + d).detach(), rope, positions, axes).double() for d in (step, -step))
        slope = float(((up - down) * w.double()).sum())
        # each of two elements of either output is off by 4 roundings of at most |x| + 1, and weighed
        bound = 4 * 4 * 2.0 ** -24 * float(x.detach().abs().max() + 1) * 2 * float(w.abs().max())
        assert abs(slope - float(x.grad[at])) <= bound


def test_shapes_broadcasts_and_second_derivatives():
    rope, axes = wht.wht_attention_rope_table(40, 64, device=DEV), wht.wht_rotary_axes((16, 16))
    x = torch.randn(2, 15, 3, 64, device=DEV, requires_grad=True)
    positions = torch.randint(0, 40, (2, 15, 2), dtype=torch.int32, device=DEV)
    y = wht_rotary(x, rope, positions, axes)
    flat = wht.wht_rotary_rotate(x.detach().view(30, 3, 64), rope, positions.view(30, 2), axes)
    assert torch.equal(y.detach().view(30, 3, 64), flat)
    assert torch.equal(wht_rotary(x.detach(), rope, positions[..., 0]), wht_rotary(x.detach(), rope, positions[..., 0].unsqueeze(-1)))
    dx, = torch.autograd.grad(y.sum(), x, create_graph=True)         # a gradient of ones that all stand in one place
    ones = wht.wht_rotary_rotate(torch.ones(30, 3, 64, device=DEV), rope, positions.view(30, 2), axes, inverse=True)
    assert torch.equal(dx.detach().view(30, 3, 64), ones)
    dy = torch.randn_like(x).requires_grad_(True)
    dx, = torch.autograd.grad(wht_rotary(x, rope, positions, axes), x, dy, create_graph=True)
    v = torch.randn_like(x)
    again, = torch.autograd.grad(dx, dy, v)                          # of R^T dy by dy: R v
    assert torch.equal(again, wht_rotary(v, rope, positions, axes))
    shared = torch.randn(15, 1, 64, device=DEV, requires_grad=True)  # one head for all: its gradient is their sum
    y = wht_rotary(shared.expand(15, 3, 64), rope, positions[0].contiguous(), axes)
    w = torch.randn_like(y)
    g, = torch.autograd.grad(y, shared, w)
    parts = wht.wht_rotary_rotate(w, rope, positions[0].contiguous(), axes, inverse=True)
    assert float((g - parts.sum(1, keepdim=True)).abs().max()) < 1e-5
    odd = torch.randn(15, 3, 65, device=DEV)[:, :, 1:].requires_grad_(True)            # not 16-byte steps
    y = wht_rotary(odd, rope, positions[0].contiguous(), axes)
    assert torch.equal(y, wht_rotary(odd.detach().clone(), rope, positions[0].contiguous(), axes))
    with pytest.raises(ValueError, match="positions must be those"):
        wht_rotary(x, rope, positions[:, :3], axes)


def test_without_positions_or_axes():
    rope = wht.wht_attention_rope_table(40, 64, device=DEV)
    x = torch.randn(15, 3, 64, device=DEV, requires_grad=True)
    y = wht_rotary(x, rope)
    assert torch.equal(y.detach(), wht.wht_rotary_rotate(x.detach(), rope))
    dy = torch.randn_like(y)
    assert torch.equal(torch.autograd.grad(y, x, dy)[0], wht.wht_rotary_rotate(dy, rope, inverse=True))
    dy.requires_grad_(True)
    dx, = torch.autograd.grad(wht_rotary(x, rope), x, dy, create_graph=True)
    assert torch.equal(torch.autograd.grad(dx, dy, x.detach())[0], y)
    listed = wht_rotary(x, rope, torch.arange(15, dtype=torch.int32, device=DEV), axes=[0] * 32)
    assert torch.equal(listed, y)


def test_changed_angles_raise():
    x, positions, rope = make(4, 2, 32, 32, (8, 8), F32)
    y = wht_rotary(x.requires_grad_(True), rope, positions, wht.wht_rotary_axes((8, 8)))
    positions += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def captured_step(x, positions, rope, axes, dy):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(wht_rotary(x, rope, positions, axes), x, dy)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = wht_rotary(x, rope, positions, axes)
        dx, = torch.autograd.grad(y, x, dy)
    return graph, y.detach(), dx


def test_captured_training_step():
    """Forward and gradient in a graph; replays follow the inputs, with eager work between."""
    x, positions, rope = make(64, 4, 64, 64, (8, 12, 12), B16)
    axes = wht.wht_rotary_axes((8, 12, 12))
    x.requires_grad_(True)
    dy = torch.randn(64, 4, 64, device=DEV).to(B16)
    graph, y, dx = captured_step(x, positions, rope, axes, dy)
    for _ in range(3):
        with torch.no_grad():
            x.normal_()
        dy.normal_()
        positions.random_(0, 40)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, wht.wht_rotary_rotate(x.detach(), rope, positions, axes))
        assert torch.equal(dx, wht.wht_rotary_rotate(dy, rope, positions, axes, inverse=True))


def test_a_leaf_of_a_living_graph_is_refused_in_a_capture():
    x, positions, rope = make(64, 4, 64, 64, (8, 12, 12), B16)
    axes = wht.wht_rotary_axes((8, 12, 12))
    x.requires_grad_(True)
    alive = wht_rotary(x, rope, positions, axes)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError, match="let go of that graph"):
            wht_rotary(x, rope, positions, axes)
        out = wht_rotary(x.detach(), rope, positions, axes)          # without a gradient it is taken
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, alive)


@pytest.mark.parametrize("plain", [True, False])
def test_the_gradient_is_the_same_on_either_path(plain, monkeypatch):
    """A node of C++ autograd, and the Python Function."""
    x, positions, rope = make(20, 4, 64, 32, (4, 6, 6), B16)
    axes = wht.wht_rotary_axes((4, 6, 6))
    if not plain:
        monkeypatch.setattr(attention4, "_native_module", attention4._NoNative)
    x.requires_grad_(True)
    y = wht_rotary(x, rope, positions, axes, True)
    assert ("WhtRotaryFunction" in type(y.grad_fn).__name__ + str(y.grad_fn.name())) and y.grad_fn.next_functions[0][0] is not None
    dy = torch.randn(20, 4, 64, device=DEV).to(B16)
    dx, = torch.autograd.grad(y, x, dy)
    assert torch.equal(dx, wht.wht_rotary_rotate(dy, rope, positions, axes, True, inverse=True))


def test_results_do_not_depend_on_the_way_the_call_is_marshalled(monkeypatch):
    x, positions, rope = make(33, 4, 64, 32, (4, 6, 6), B16)
    axes = wht.wht_rotary_axes((4, 6, 6))
    native = [wht.wht_rotary_rotate(x, rope, positions, axes, interleaved=i, inverse=j) for i in (False, True) for j in (False, True)]
    monkeypatch.setattr(attention4, "_native_module", attention4._NoNative)
    other = [wht.wht_rotary_rotate(x, rope, positions, axes, interleaved=i, inverse=j) for i in (False, True) for j in (False, True)]
    assert all(torch.equal(a, b) for a, b in zip(native, other))


def test_refusals_name_the_argument():
    x, positions, rope = make(4, 2, 64, 64, (16, 16), B16)
    for match, kw in (("x must be", dict(x=x[0])), ("rope must be", dict(rope=rope.double())), ("positions must be", dict(positions=positions.long())),
                      ("positions must be", dict(positions=positions[:3])), ("one number for each", dict(axes=bytes(5))), ("axes must be below 2", dict(axes=bytes([2] * 32))),
                      ("out must match", dict(out=x.float()))):
        with pytest.raises(ValueError, match=match):
            wht.wht_rotary_rotate(**{"x": x, "rope": rope, "positions": positions, **kw})
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        wht.wht_rotary_rotate(x.half(), rope, positions)
    for kw in (dict(x=torch.randn(4, 2, 72, device=DEV)), dict(rope=rope[:, :12].contiguous()), dict(x=torch.randn(4, 2, 272, device=DEV)),
               dict(out=torch.empty(1, 2, 64, dtype=B16, device=DEV).expand(4, 2, 64)), dict(x=torch.randn(4, 2, 65, device=DEV).to(B16)[:, :, 1:])):
        with pytest.raises(wht.WhtRotaryError, match="status"):
            wht.wht_rotary_rotate(**{"x": x, "rope": rope, **kw})
    assert wht.wht_rotary_rotate(x[:0], rope, positions[:0]).shape == (0, 2, 64)
    assert WhtRotaryFunction.apply(x, rope, positions, None, False, False).shape == x.shape and math.isfinite(float(x.float().sum()))
