"""autograd.wht_rotary as a node of torch's C++ autograd (csrc/attention_marshal.cpp) against the Python Function that it stands for: values bit for
bit, and the same answer -- a result or an error -- under every mode that looks into an autograd function, and for whatever a graph's hooks
make of the table and the positions that it saved."""
import numpy as np
import pytest
import torch

import paper_2603_08343_amd as wht
from paper_2603_08343_amd import attention4
from paper_2603_08343_amd.autograd import wht_rotary

pytestmark = pytest.mark.gpu

T, H, D, ROWS = 24, 3, 64, 40
AXES = wht.wht_rotary_axes((6, 5, 5))


def _tensors(dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(4)
    x, dy = (torch.empty(T, H, D, device="cuda", dtype=dtype).normal_(generator=g) for _ in range(2))
    positions = torch.randint(0, ROWS, (T, 3), device="cuda", generator=g).to(torch.int32)
    return x, dy, wht.wht_attention_rope_table(ROWS, 32), positions


def _flat(out):
    out = out if isinstance(out, (tuple, list)) else (out,)
    return [t if not isinstance(t, torch.Tensor) else (t.dtype, tuple(t.shape), t.requires_grad, t.detach().double().cpu()) for t in out]


def _outcome(call):
    try:
        out = _flat(call())
        torch.cuda.synchronize()
        return out
    except Exception as e:                                           # compared, not hidden
        text = str(e)
        for node in ("torch::autograd::CppNode<WhtRotaryFunction>", "WhtRotaryFunctionBackward"):
            text = text.replace(node, "node")
        return type(e), text


def _same(call, monkeypatch, label, fails=None):
    """call() builds everything it needs: it runs once on each path.  fails: what it has to raise."""
    print(f"[rotary] {label}", flush=True)
    native, module = _outcome(call), attention4._native()

    class NoNode:
        append4, paged4, rotate, leaf_elsewhere = (staticmethod(getattr(module, n)) for n in ("append4", "paged4", "rotate", "leaf_elsewhere"))
        rotary = staticmethod(lambda *args: None)

    with monkeypatch.context() as m:
        m.setattr(attention4, "_native_module", NoNode)
        general = _outcome(call)
    if isinstance(general, tuple):
        assert native == general, label
        assert fails is None or general[0] is fails, general
        return
    assert fails is None, (label, general)
    assert isinstance(native, list) and len(native) == len(general), (label, native)
    for n, g in zip(native, general):
        if isinstance(n, tuple) and isinstance(n[-1], torch.Tensor):
            assert n[:3] == g[:3] and torch.equal(n[3].nan_to_num(7.0), g[3].nan_to_num(7.0)), label
        else:
            assert n == g, label


def _train(dtype=torch.bfloat16, positions=True, axes=True, again=False):
    x, dy, rope, p = _tensors(dtype)
    x.requires_grad_(True)
    if again:
        dy.requires_grad_(True)
    y = wht_rotary(x, rope, p if positions else None, AXES if axes else None)
    dx, = torch.autograd.grad(y, x, dy, create_graph=again)
    return (y, dx, *torch.autograd.grad(dx, dy, x.detach())) if again else (y, dx)


def test_the_node_takes_plain_calls_and_declines_the_others():
    x, _, rope, p = _tensors()
    node = attention4._native().rotary
    for ok in ((x, rope, p, AXES), (x.float(), rope, p, None), (x, rope, None, None), (x.view(2, 12, H, D), rope, p, AXES), (torch.nn.Parameter(x), rope, p, AXES)):
        assert node(*ok, False) is not None
    for other in ((x.half(), rope, p, AXES), (x.cpu(), rope, p, AXES), (x, rope.double(), p, AXES), (x, rope, p.long(), AXES), (x, rope, p[:5], AXES), (x, rope, p, list(AXES)),
                  (x, rope, None, AXES), (x[:0], rope, p[:0], AXES), (x[..., :40], rope, p, AXES), (x, rope[:, ::2], p, None), (None, rope, p, AXES), (x, None, p, AXES)):
        assert node(*other, False) is None
    with torch.autograd.forward_ad.dual_level():
        assert node(x, rope, p, AXES, False) is None
    with torch.overrides.TorchFunctionMode():
        assert node(x, rope, p, AXES, False) is None


@pytest.mark.parametrize("again", [False, True])
def test_saved_tensors_that_a_hook_changed(again, monkeypatch):
    """The backward pass reads the table and the positions where a hook left them: another type, place, shape or stride is refused as it is of a call."""
    def hooked(change, **kw):
        def call():
            with torch.autograd.graph.saved_tensors_hooks(lambda t: t, change):
                return _train(again=again, **kw)
        return call

    table = lambda f: lambda t: f(t) if t.is_floating_point() and t.dim() == 3 and t.shape[-1] == 2 else t
    places = lambda f: lambda t: f(t) if t.dtype == torch.int32 else t
    for label, f in (("half", lambda t: t.half()), ("double", lambda t: t.double()), ("cpu", lambda t: t.cpu()), ("flat", lambda t: t.flatten()), ("narrow", lambda t: t[:, :8]),
                     ("stepped", lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)), ("one number a pair", lambda t: t[..., :1].contiguous())):
        _same(hooked(table(f)), monkeypatch, f"table {label}", ValueError)
    _same(hooked(table(lambda t: t[:, :8].contiguous())), monkeypatch, "a narrower table than the axes", ValueError)
    for label, f in (("long", lambda t: t.long()), ("cpu", lambda t: t.cpu()), ("fewer", lambda t: t[:5].contiguous()), ("stepped", lambda t: t.t().contiguous().t()),
                     ("empty", lambda t: t[:0]), ("five axes", lambda t: torch.cat((t, t[:, :2]), 1)), ("bytes", lambda t: t.to(torch.uint8)),
                     ("fewer axes than pairs name", lambda t: t[:, :2].contiguous())):
        _same(hooked(places(f)), monkeypatch, f"positions {label}", ValueError)
    # what a call takes is taken: fewer rows (positions past them give NaN), a narrower table without axes, other angles
    _same(hooked(table(lambda t: t[:7].contiguous())), monkeypatch, "fewer rows")
    _same(hooked(table(lambda t: t[:0])), monkeypatch, "no rows")
    _same(hooked(table(lambda t: t[:, :8].contiguous()), axes=False), monkeypatch, "a narrower table")
    _same(hooked(table(lambda t: t * 2), positions=False, axes=False), monkeypatch, "another table")
    _same(hooked(places(lambda t: t // 2)), monkeypatch, "other positions")
    _same(hooked(places(lambda t: t[:, 0].contiguous()), axes=False), monkeypatch, "one axis")


def test_modes_hooks_and_transforms(monkeypatch):
    x, dy, rope, p = _tensors()

    def under(ctx, **kw):
        with ctx:
            return _train(**kw)

    def hooks():
        seen = []
        with torch.autograd.graph.saved_tensors_hooks(lambda t: seen.append((tuple(t.shape), t.dtype)) or t.cpu(), lambda t: t.cuda()):
            out = _train()
        return (*out, tuple(seen))

    def checkpointed():
        x, dy, rope, p = _tensors()
        y = torch.utils.checkpoint.checkpoint(lambda t: wht_rotary(t, rope, p, AXES), x.requires_grad_(True), use_reentrant=False)
        return (y, *torch.autograd.grad(y, x, dy))

    def forward_mode():
        with torch.autograd.forward_ad.dual_level():
            return wht_rotary(torch.autograd.forward_ad.make_dual(x, dy), rope, p, AXES)

    def no_grad():
        with torch.no_grad():
            return wht_rotary(x.clone().requires_grad_(True), rope, p, AXES)

    def inference():
        with torch.inference_mode():
            y = wht_rotary(x, rope, p, AXES)
            return y, y.is_inference()

    def inference_saved():
        with torch.inference_mode():
            t = rope.clone()
        return wht_rotary(x.clone().requires_grad_(True), t, p, AXES)

    def twice(retain):
        x, dy, rope, p = _tensors()
        y = wht_rotary(x.requires_grad_(True), rope, p, AXES)
        return (*torch.autograd.grad(y, x, dy, retain_graph=retain), *torch.autograd.grad(y, x, dy))

    def result_changed(shape):
        x, dy, rope, p = _tensors()
        y = wht_rotary(x.requires_grad_(True).view(shape), rope, p.view(*shape[:-2], 3), AXES)
        y.add_(1.0)
        y[0].zero_()
        return (y, y._base is None, *torch.autograd.grad(y, x, dy.view(shape)))

    def table_changed():
        x, dy, rope, p = _tensors()
        y = wht_rotary(x.requires_grad_(True), rope, p, AXES)
        rope.mul_(2.0)
        return torch.autograd.grad(y, x, dy)

    def side_stream():
        side, fill = torch.cuda.Stream(), torch.empty(1 << 28, device="cuda")
        late = torch.zeros_like(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            fill.zero_()
            late.copy_(x)
            late.requires_grad_(True)
            y = wht_rotary(late, rope, p, AXES)
            out = (y, *torch.autograd.grad(y, late, dy))
        torch.cuda.synchronize()
        return out

    for again in (False, True):
        for dtype in (torch.bfloat16, torch.float32):
            _same(lambda: _train(dtype, again=again), monkeypatch, f"{dtype} again={again}")
    _same(hooks, monkeypatch, "saved tensor hooks")
    _same(checkpointed, monkeypatch, "checkpoint")
    _same(lambda: under(torch.autocast("cuda", dtype=torch.bfloat16)), monkeypatch, "autocast")
    _same(lambda: under(torch.autograd.detect_anomaly(check_nan=False)), monkeypatch, "anomaly mode")
    _same(lambda: under(torch.overrides.TorchFunctionMode()), monkeypatch, "function mode")
    _same(forward_mode, monkeypatch, "forward mode")
    _same(no_grad, monkeypatch, "no_grad")
    _same(inference, monkeypatch, "inference mode")
    _same(inference_saved, monkeypatch, "inference tensor to be saved")
    _same(lambda: twice(True), monkeypatch, "retained graph")
    _same(lambda: twice(False), monkeypatch, "freed graph")
    for shape in ((T, H, D), (2, T // 2, H, D)):
        _same(lambda: result_changed(shape), monkeypatch, f"result changed in place, {shape}")
    _same(table_changed, monkeypatch, "table changed in place")
    _same(side_stream, monkeypatch, "side stream")
    _same(lambda: torch.vmap(lambda t: wht_rotary(t, rope, p, AXES))(torch.stack((x, x))), monkeypatch, "vmap")
    _same(lambda: torch.vmap(lambda s: wht_rotary(x, rope, p, AXES) * s)(torch.ones(2, device="cuda", dtype=x.dtype)), monkeypatch, "vmap, captured tensors")
    _same(lambda: torch.func.grad(lambda t: wht_rotary(t, rope, p, AXES).float().sum())(x), monkeypatch, "func.grad")
    _same(lambda: torch.func.jvp(lambda t: wht_rotary(t, rope, p, AXES), (x,), (dy,)), monkeypatch, "func.jvp")


def test_gradients_of_any_layout(monkeypatch):
    def graded(form):
        x, dy, rope, p = _tensors()
        y = wht_rotary(x.requires_grad_(True), rope, p, AXES)
        return torch.autograd.grad(y, x, form(dy))

    _same(lambda: graded(lambda dy: dy.transpose(0, 1).contiguous().transpose(0, 1)), monkeypatch, "heads outside")
    _same(lambda: graded(lambda dy: dy[:, :1].expand(T, H, D)), monkeypatch, "one head's for all")
    _same(lambda: graded(lambda dy: dy[:1, :1, :1].expand(T, H, D)), monkeypatch, "one number for all")
    _same(lambda: graded(lambda dy: torch.cat((dy, dy), -1)[..., 1:D + 1]), monkeypatch, "not in 16-byte steps")
    _same(lambda: graded(lambda dy: dy.float()), monkeypatch, "float32 gradient of a bfloat16 result")


def test_threads():
    """Backward passes of several graphs at once: each on its own tensors, all equal to the Python Function's."""
    import concurrent.futures
    x, dy, rope, p = _tensors()
    want = wht.wht_rotary_rotate(x, rope, p, AXES), wht.wht_rotary_rotate(dy, rope, p, AXES, inverse=True)

    def one(_):
        for _ in range(20):
            t = x.detach().clone().requires_grad_(True)
            y = wht_rotary(t, rope, p, AXES)
            if not (torch.equal(y, want[0]) and torch.equal(torch.autograd.grad(y, t, dy)[0], want[1])):
                return False
        return True

    with concurrent.futures.ThreadPoolExecutor(4) as pool:
        assert all(pool.map(one, range(8)))


def test_compiled_autograd_of_a_graph_built_eagerly():
    compiled_autograd = pytest.importorskip("torch._dynamo.compiled_autograd")
    x, dy, rope, p = _tensors()
    x.requires_grad_(True)
    want, = torch.autograd.grad(wht_rotary(x, rope, p, AXES), x, dy)
    y = wht_rotary(x, rope, p, AXES)
    with compiled_autograd._enable(torch.compile(backend="eager")):
        y.backward(dy)
    assert torch.equal(x.grad, want)


@pytest.mark.parametrize("without", [torch.no_grad, torch.inference_mode])
def test_a_capture_without_a_gradient_takes_any_leaf(without):
    """Of a leaf that a living graph holds a capture is refused where it records a gradient; without one there is nothing to wait for."""
    x, _, rope, p = _tensors()
    x.requires_grad_(True)
    alive = wht_rotary(x, rope, p, AXES)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with without():
            y = wht_rotary(x, rope, p, AXES)
        with pytest.raises(RuntimeError, match="let go of that graph"):
            wht_rotary(x, rope, p, AXES)
    for _ in range(3):
        with torch.no_grad():
            x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, wht.wht_rotary_rotate(x.detach(), rope, p, AXES))
    assert alive.requires_grad and not y.requires_grad


@pytest.mark.parametrize("lead", [(1,), (3,), (2, 2), (0,), (1, 4)], ids=str)
def test_without_positions_tokens_count_within_their_batch(lead, monkeypatch):
    """x [..., tokens, heads, head_dim]: each batch begins at 0, and a table of as many rows as it has tokens is long enough."""
    n = 10
    rope = wht.wht_attention_rope_table(n, 32)
    g = torch.Generator(device="cuda").manual_seed(6)
    x, dy = (torch.empty(*lead, n, H, D, device="cuda").normal_(generator=g) for _ in range(2))
    want = [torch.stack([wht.wht_rotary_rotate(t, rope, inverse=back) for t in u.reshape(-1, n, H, D)]).view(u.shape) if u.numel() else u
            for u, back in ((x, False), (dy, True))]

    def call():
        t = x.clone().requires_grad_(True)
        y = wht_rotary(t, rope)
        dx, = torch.autograd.grad(y, t, dy)
        assert torch.equal(y, want[0]) and torch.equal(dx, want[1]) and not torch.isnan(y).any()
        return y, dx

    call()
    _same(call, monkeypatch, f"no positions, {lead}")


@pytest.mark.parametrize("kind", [list, iter, lambda a: np.array(list(a), dtype=np.int16), torch.tensor], ids=["list", "iterator", "array", "tensor"])
def test_axes_of_any_kind_are_those_of_the_call(kind):
    """The backward pass turns back by the axes that the call had, whatever became of them."""
    x, dy, rope, p = _tensors()
    want = wht.wht_rotary_rotate(x, rope, p, AXES), wht.wht_rotary_rotate(dy, rope, p, AXES, inverse=True)
    axes = kind(list(AXES))
    y = wht_rotary(x.requires_grad_(True), rope, p, axes)
    if hasattr(axes, "__setitem__"):
        axes[3] = 1
    assert torch.equal(y, want[0]) and torch.equal(torch.autograd.grad(y, x, dy)[0], want[1])
    c = [t.cuda() for t in (torch.zeros(2, 1, 16, 32, dtype=torch.uint8), torch.zeros(2, 1, 16, 2, dtype=torch.uint8))]
    table, lengths, k = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda"), torch.randn(1, 1, D, device="cuda")
    q = [wht.wht_attention_append4(k, k, k, c[0], c[0].clone(), c[1], c[1].clone(), table, lengths, rope, positions=p[:1], axes=a) for a in (AXES, kind(list(AXES)))]
    assert torch.equal(*q)


def test_under_a_compilers_trace():
    """The trace breaks at the call, which goes to the Python Function: values and gradients of the eager call."""
    x, dy, rope, p = _tensors()
    x.requires_grad_(True)
    y = wht_rotary(x * 2, rope, p, AXES) + 1
    want, = torch.autograd.grad(y, x, dy)
    compiled = torch.compile(lambda t: wht_rotary(t * 2, rope, p, AXES) + 1, backend="eager")
    for _ in range(2):
        z = compiled(x)
        assert torch.equal(z, y) and torch.equal(torch.autograd.grad(z, x, dy)[0], want)
    batch = torch.compile(lambda t: wht_rotary(t, rope), backend="eager")
    assert torch.equal(batch(x.detach().view(2, 12, H, D)), wht_rotary(x.detach().view(2, 12, H, D), rope))
