"""Calls of the gated recurrence that a program makes at its edges: no segments, rows that none has, torch's other modes and hooks."""
import ctypes as C

import numpy as np
import pytest
import torch
import torch.utils.checkpoint

import paper_1804_10727_amd as idf
from oracle import few_bits as oracle
from paper_1804_10727_amd import tokens

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
W = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def make(n, channels, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return tuple((torch.randn(n, channels, generator=g) * f + o).to(dtype).to(DEV) for f, o in ((1, 0), (2, 3), (1, 0)))


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,channels", [(1, 1), (300, 70), (5000, 130)])
def test_gradients_without_segments(rows, channels, dtype):
    """None of the segments has a row where there are no segments: gradients are zero, by the library's own call as by the tensors'."""
    x, gates, d = make(rows, channels, dtype)
    offsets = torch.zeros(1, dtype=torch.int64, device=DEV)
    dx, dg = (torch.full_like(x, float("nan")) for _ in range(2))
    kept = torch.full((3, channels), 5.0, device=DEV)
    r = [tokens._as_rows(t) for t in (x, gates, d, dx, dg)]
    a = tokens._GateScanBackward(int(dtype == torch.bfloat16), channels, rows, rows, 0, 3, *r, None, kept.data_ptr(), None, offsets.data_ptr(), None, None, 0)
    assert idf.load_library().idf_gate_scan_backward(C.byref(a), C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    torch.cuda.synchronize()
    assert not dx.any() and not dg.any() and torch.all(kept == 5.0)
    marks = torch.empty((rows // 16 + 1) * channels, device=DEV)
    for f in (idf.gate_scan_backward, lambda *args, **kw: tokens._gate_scan_backward(*args, None, **kw, n_segments=None, stream_ids=None, n_streams=3)):
        filler = [torch.full_like(x, float("nan")) for _ in range(2)]
        del filler                                 # (their memory is likely to be taken for the gradients)
        got = f(x, gates, marks, d, offsets=offsets, max_tokens=rows)
        assert not got[0].any() and not got[1].any() and not got[2].any()
    leaves = [t.clone().requires_grad_() for t in (x, gates)]
    out, ends = idf.gate_scan_recorded(*leaves, offsets=offsets, max_tokens=rows)
    assert not out.any() and ends.shape == (0, channels)
    out.backward(d)
    assert not leaves[0].grad.any() and not leaves[1].grad.any()


def test_tangents_are_refused():
    """Forward mode: refused by every call, not answered with a derivative of zero; what carries no tangent is taken beside it."""
    x, gates, d = make(40, 64, torch.float32)
    w, ws = idf.quantize_rows(torch.randn(32, 64, device=DEV))
    ring, heads = idf.nibble_ring(1, 64, 1, 64, DEV), x[:, None]
    _, marks = idf.gate_scan(x, gates, marks=True)
    state = torch.zeros(1, 64, device=DEV)
    with torch.autograd.forward_ad.dual_level():
        t = torch.autograd.forward_ad.make_dual(x, torch.ones_like(x))
        h = t[:, None]
        for call in (lambda: idf.gate_scan(t, gates), lambda: idf.gate_scan(x, t), lambda: idf.gate_scan(x, gates, t[:1]), lambda: idf.gate_scan_backward(x, gates, marks, t), lambda: idf.quantize_rows(t),
                     lambda: idf.project_rows(t, w, ws), lambda: idf.project_rows(x, w, ws, bias=t[0, :32]), lambda: idf.nibble_append(h, heads, ring), lambda: idf.nibble_attend(h, ring, window=9),
                     lambda: idf.norm_rotate(h, heads, torch.arange(40, device=DEV), idf.rotary_frequencies(64, device=DEV)[0]), lambda: idf.window_attend(heads, h, heads, window=9),
                     lambda: idf.decay_attend(heads, heads, h, torch.zeros(1, device=DEV))):
            for mode in (torch.enable_grad, torch.no_grad):
                with mode(), pytest.raises(ValueError, match="tangent"):
                    call()
        with pytest.raises((NotImplementedError, RuntimeError)):
            idf.gate_scan_recorded(t, gates, state)
        assert torch.equal(idf.gate_scan(x, gates, state), idf.gate_scan(t.detach(), gates, state))
        with torch.autograd.forward_ad._set_fwd_grad_enabled(False):
            assert torch.equal(idf.gate_scan(t, gates, state), idf.gate_scan(x, gates, state))


@pytest.mark.parametrize("call", [lambda x, g: idf.gate_scan(x, g), lambda x, g: idf.gate_scan_recorded(x, g)[0]], ids=["gate_scan", "recorded"])
def test_torchs_transforms_are_refused(call):
    """vmap, grad and jvp hand over tensors without memory of their own."""
    x, gates, _ = make(40, 64, torch.float32)
    for f in (lambda: torch.func.vmap(call)(x[None], gates[None]), lambda: torch.func.grad(lambda y: call(y, gates).sum())(x), lambda: torch.func.jvp(lambda y: call(y, gates), (x,), (x,))):
        with pytest.raises((RuntimeError, ValueError, NotImplementedError)):
            f()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("channels", [64, 33])
@pytest.mark.parametrize("offsets,longest", [([0], 1), ([3, 4, 4, 9], 5), ([0, 100, 300], 60), ([7, 250, 250, 600], 250), ([300, 1000, 1000, 4000], 2500), ([100, 9000, 30000], 20000), ([0, 40], 0)], ids=str)
def test_new_results_are_zero_where_no_segment_is(offsets, longest, channels, dtype):
    """In front of, behind and between segments, and beyond max_tokens: what a call makes itself holds zeros there, recorded or not; what is given stays."""
    n = offsets[-1] + 700
    x, gates, d = make(n, channels, dtype, seed=n)
    kw = dict(offsets=torch.tensor(offsets, device=DEV), max_tokens=longest)
    mine = torch.zeros(n, dtype=torch.bool)
    for a, b in zip(offsets, offsets[1:]):
        mine[a:min(b, a + longest)] = True
    given = torch.full_like(x, 7.0)
    idf.gate_scan(x, gates, out=given, **kw)
    assert torch.all(given[~mine] == 7.0)
    leaf = x.clone().requires_grad_()
    long = tokens._make_recorded().apply
    for call in (lambda: idf.gate_scan(x, gates, **kw), lambda: tokens._gate_scan(x, gates, None, None, kw["offsets"], longest, None, None, None, None), lambda: idf.gate_scan(x, gates, marks=True, **kw)[0],
                 lambda: idf.gate_scan_recorded(leaf, gates, **kw)[0], lambda: long(leaf, gates, None, kw["offsets"], longest, None)[0]):
        filler = torch.full_like(x, float("nan"))
        del filler                                 # (its memory is likely to be taken for the result)
        got = call().detach()
        assert not got[~mine].any() and torch.equal(got[mine], given[mine])


def test_padding_multiplied_away_leaves_no_nan():
    """A loss over a padded batch, its padding masked by multiplication."""
    x, gates, d = make(2000, 64, torch.float32, seed=3)
    filler = [torch.full_like(x, float("nan")) for _ in range(4)]
    del filler
    leaf = x.clone().requires_grad_()
    out, ends = idf.gate_scan_recorded(leaf, gates, offsets=torch.tensor([0, 500, 900], device=DEV), max_tokens=500)
    mask = torch.zeros(2000, 1, device=DEV)
    mask[:900] = 1
    ((out * mask * d).sum() + ends.sum()).backward()
    assert torch.isfinite(leaf.grad).all() and not leaf.grad[900:].any() and leaf.grad[:900].any(1).all()


def recorded(dtype, lengths=(300, 0, 45)):
    x, gates, d = make(sum(lengths), 66, dtype, seed=5)
    kw = dict(offsets=torch.tensor([0] + list(lengths)).cumsum(0).to(DEV), max_tokens=max(lengths))
    leaves = [t.clone().requires_grad_() for t in (x, gates)] + [torch.randn(len(lengths), 66, generator=torch.Generator().manual_seed(6)).to(DEV).requires_grad_()]
    out, ends = idf.gate_scan_recorded(*leaves, **kw)
    torch.autograd.backward([out, ends], [d, torch.ones_like(ends)])
    return leaves, kw, d, [t.grad for t in leaves]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_saved_tensors_by_way_of_hooks(dtype):
    """Kept on the host, or laid out anew, in the meantime: the same gradients.  Of another type or size when they come back: an error of torch's, nothing is read."""
    leaves, kw, d, want = recorded(dtype)

    def again(hooks):
        mine = [t.detach().clone().requires_grad_() for t in leaves]
        with hooks:
            out, ends = idf.gate_scan_recorded(*mine, **kw)
        torch.autograd.backward([out, ends], [d, torch.ones_like(ends)])
        return [t.grad for t in mine]
    hooks = torch.autograd.graph.saved_tensors_hooks
    for keep in (torch.autograd.graph.save_on_cpu(), hooks(lambda t: t.clone(), lambda t: t), hooks(lambda t: t, lambda t: t.t().contiguous().t() if t.dim() == 2 and t.shape[1] == 1 else t.clone())):
        assert all(torch.equal(a, b) for a, b in zip(again(keep), want))
    for change in (lambda t: t.half() if t.dim() == 2 else t, lambda t: t[:-1] if t.dim() == 2 else t, lambda t: t[:, :-2].contiguous() if t.dim() == 2 else t, lambda t: t.cpu(),
                   lambda t: t[:-1] if t.dtype == torch.int64 else t, lambda t: t.int() if t.dtype == torch.int64 else t, lambda t: t[:5] if t.dim() == 1 and t.is_floating_point() else t):
        with pytest.raises(RuntimeError):
            again(hooks(lambda t: t, change))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("reentrant", [False, True])
def test_checkpointed(dtype, reentrant):
    leaves, kw, d, want = recorded(dtype)
    mine = [t.detach().clone().requires_grad_() for t in leaves]
    out, ends = torch.utils.checkpoint.checkpoint(lambda *a: idf.gate_scan_recorded(*a, **kw), *mine, use_reentrant=reentrant)
    torch.autograd.backward([out, ends], [d, torch.ones_like(ends)])
    assert all(torch.equal(t.grad, w) for t, w in zip(mine, want))


def test_errors_of_hooks_are_the_programs():
    class Stop(Exception):
        pass

    def stop(t):
        raise Stop
    x, gates, _ = make(40, 64, torch.float32)
    leaf = x.clone().requires_grad_()
    with torch.autograd.graph.saved_tensors_hooks(stop, lambda t: t), pytest.raises(Stop):
        idf.gate_scan_recorded(leaf, gates)
    out, _ = idf.gate_scan_recorded(leaf, gates)
    out.sum().backward()
    assert torch.isfinite(leaf.grad).all()


def test_two_checkpoints_behind_each_other():
    """A stack of two layers, each run again for its gradients, some of the leaves shared."""
    x, gates, d = make(700, 64, torch.float32, seed=9)
    kw = dict(offsets=torch.tensor([0, 300, 700], device=DEV), max_tokens=400)

    def layer(h, g, w):
        return idf.gate_scan_recorded(torch.tanh(h * w), g * w, **kw)[0]
    grads = []
    for run in (lambda f, *a: f(*a), lambda f, *a: torch.utils.checkpoint.checkpoint(f, *a, use_reentrant=False)):
        a, g, w = (t.clone().requires_grad_() for t in (x, gates, torch.linspace(0.5, 1.5, 64, device=DEV)))
        run(layer, run(layer, a, g, w), g, w).backward(d)
        grads.append([t.grad for t in (a, g, w)])
    assert all(torch.equal(p, q) for p, q in zip(*grads))


def test_leaves_changed_before_the_backward_pass_are_refused():
    leaves, kw, d, _ = recorded(torch.float32)
    x, gates = leaves[0].detach().clone().requires_grad_(), leaves[1].detach().clone()
    out, _ = idf.gate_scan_recorded(x, gates, **kw)
    gates += 1
    with pytest.raises(RuntimeError, match="modified"):
        out.backward(d)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("n", [5, 40, 3000])
def test_states_and_values_far_apart(n, dtype):
    """Values near the largest number, of either sign: a difference between a state and a value goes beyond it, what gates make of that does not.  Where it flows
    into no gradient there is none, and not what is no number."""
    g = torch.Generator().manual_seed(n)
    x, gates = torch.randn(n, 64, generator=g).to(dtype), (torch.randn(n, 64, generator=g) + 1).to(dtype)
    d, state = torch.zeros(n, 64, dtype=dtype), torch.randn(1, 64, generator=g)
    big = 3.2e38
    x[n // 2, 3], state[0, 3] = big, -big
    x[n - 1, 7], x[n - 2, 7] = -big, big
    x[:, 11] = torch.where(torch.arange(n) % 2 == 0, big, -big).to(dtype)
    d[:, 20:] = torch.randn(n, 44, generator=g).to(dtype)
    x[n // 3, 30], x[n // 3 + 1, 30], d[:, 30] = big, -big, (d[:, 30].float() * 1e-30).to(dtype)
    end = torch.zeros(1, 64)
    out, marks = idf.gate_scan(x.to(DEV), gates.to(DEV), state.to(DEV), marks=True)
    got = idf.gate_scan_backward(x.to(DEV), gates.to(DEV), marks, d.to(DEV), end.to(DEV))
    hs, _, errors = oracle.gate_scan(f64(x), f64(gates), f64(state[0]))
    dx, dg, ds, ex, eg, es = oracle.gate_scan_backward(f64(x), f64(gates), f64(state[0]), f64(d), f64(end[0]))
    u = torch.finfo(dtype).eps / 2
    # (a gradient here is the difference of two products that are rounded once more: 2 W of their sizes, which eg, of them and their gates' errors, holds many times over)
    for t, want, bound in ((out, hs, u * np.abs(hs) + W * errors), (got[0], dx, u * np.abs(dx) + W * ex + 1e-36), (got[1], dg, u * np.abs(dg) + W * eg + 1e-36), (got[2][0], ds, W * es + 1e-30)):
        assert np.isfinite(f64(t)).all() and np.all(np.abs(f64(t) - want) <= bound)
    assert not got[1][:, :20].any() and got[1][n // 3 + 1, 30] != 0
