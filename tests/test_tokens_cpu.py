"""What the operators that mix tokens refuse, and the frequencies of a rotation: host code, no GPU needed."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_1804_10727_amd as idf
from paper_1804_10727_amd import binding, tokens
from oracle import tokens as oracle

BUF = C.create_string_buffer(4096 + 256)
AT = (C.addressof(BUF) + 255) // 256 * 256         # never read: every call below ends before anything is enqueued


def toks(stride=64, head=16, base=AT):
    return tokens._Tokens(base, stride, head)


def rotate_args(**kw):
    a = tokens._NormRotate(0, 2, 1, 16, 16, 0, 4, toks(), toks(), toks(), toks(), AT, AT, None, None, 1.0, 1e-6)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def window_args(**kw):
    a = tokens._Window(0, 2, 1, 16, 4, 4, 1, 1, 8, 8, 0, 0.25, toks(), toks(), toks(), toks(), AT, AT, None, None, None, None, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def decay_args(**kw):
    a = tokens._Decay(0, 2, 1, 16, 16, 4, 4, 1, 1, 0.25, toks(), toks(), toks(), toks(), AT, None, None, None, None, None, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def code(fn, a):
    return getattr(idf.load_library(), fn)(C.byref(a) if a is not None else None, None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw,want", [
    (dict(precision=2), -5), (dict(heads_q=-1), -1), (dict(heads_q=0, heads_k=0), -1), (dict(heads_q=5000), -1), (dict(head_dim=0), -5), (dict(head_dim=257), -5),
    (dict(rotary_dim=18), -1), (dict(rotary_dim=7), -1), (dict(rotary_dim=-2), -1), (dict(n_tokens=-1), -1), (dict(n_tokens=1 << 31), -1), (dict(eps=-1.0), -1),
    (dict(eps=NAN), -1), (dict(amplitude=INF), -1), (dict(q=toks(base=None)), -1), (dict(k_out=toks(base=None)), -1), (dict(q=toks(base=AT + 2)), -1),
    (dict(q_out=toks(head=8)), -1), (dict(k_out=toks(stride=0)), -1), (dict(positions=None), -1), (dict(frequencies=None), -1)])
def test_norm_rotate_refuses(kw, want):
    assert code("idf_norm_rotate", rotate_args(**kw)) == want and idf.load_library().idf_last_error()


@pytest.mark.parametrize("kw,want", [
    (dict(precision=2), -5), (dict(heads_q=0), -1), (dict(heads_q=3, heads_kv=2), -1), (dict(heads_kv=0), -1), (dict(head_dim=18), -5), (dict(head_dim=260), -5),
    (dict(head_dim=0), -5), (dict(n_tokens=-4), -1), (dict(max_tokens=-1), -1), (dict(n_segments=-1), -1), (dict(n_segments=2), -1), (dict(max_tokens=3), -1),
    (dict(n_streams=0), -1), (dict(n_segments=70000, n_tokens=280000, n_streams=70000), -5), (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=NAN), -1),
    (dict(scale=INF), -1), (dict(window=0), -1), (dict(sinks=-1), -1), (dict(slots=7), -1), (dict(sinks=1), -1), (dict(slots=1 << 32), -1), (dict(v_ring=None), -1),
    (dict(k_ring=AT + 8), -5), (dict(q=toks(base=None)), -1), (dict(q=toks(base=AT + 4)), -5), (dict(k=toks(stride=63)), -5), (dict(v=toks(head=18)), -5),
    (dict(out=toks(head=8)), -1), (dict(out=toks(stride=0)), -1)])
def test_window_refuses(kw, want):
    assert code("idf_window_attend", window_args(**kw)) == want and idf.load_library().idf_last_error()


@pytest.mark.parametrize("kw,want", [
    (dict(precision=7), -5), (dict(heads_q=3, heads_kv=2), -1), (dict(dim_k=18), -5), (dict(dim_k=512), -5), (dict(dim_v=2), -5), (dict(dim_v=8192), -5),
    (dict(n_tokens=5), -1), (dict(scale=NAN), -1), (dict(state_in=AT + 4), -5), (dict(state_out=AT + 8), -5), (dict(log_decay=None), -1), (dict(q=toks(base=None)), -1),
    (dict(v=toks(base=AT + 4)), -5), (dict(out=toks(stride=0)), -1)])
def test_decay_refuses(kw, want):
    assert code("idf_decay_attend", decay_args(**kw)) == want and idf.load_library().idf_last_error()


def test_decay_refuses_more_workgroups_than_a_launch_takes():
    many = dict(heads_q=1024, heads_kv=1024, n_segments=8192, n_streams=8192, n_tokens=8192, max_tokens=1)
    assert code("idf_decay_attend", decay_args(**many, dim_v=128)) == -5
    nb = C.c_size_t()
    assert idf.load_library().idf_decay_workspace(C.byref(decay_args(**many, dim_v=64)), C.byref(nb)) == 0 and nb.value == 0


def test_null_arguments_and_nothing_to_do():
    for fn in ("idf_norm_rotate", "idf_window_attend", "idf_decay_attend", "idf_window_workspace", "idf_decay_workspace"):
        assert code(fn, None) == -1
    assert code("idf_window_workspace", window_args()) == -1
    assert code("idf_norm_rotate", rotate_args(n_tokens=0)) == 0
    assert code("idf_window_attend", window_args(n_segments=0, n_tokens=0)) == 0
    assert code("idf_decay_attend", decay_args(n_tokens=0, max_tokens=0)) == 0


def test_a_workspace_that_is_too_small_is_refused():
    L = idf.load_library()
    for fn, make in (("window", lambda: window_args(heads_q=1, precision=1, head_dim=16, n_tokens=1, max_tokens=1, window=1 << 20, slots=1 << 20)),
                     ("decay", lambda: decay_args(heads_q=1, precision=1, n_tokens=1 << 20, max_tokens=1 << 20))):
        a, nb = make(), C.c_size_t()
        assert getattr(L, f"idf_{fn}_workspace")(C.byref(a), C.byref(nb)) == 0
        if nb.value:
            a.workspace, a.workspace_bytes = AT, nb.value - 1
            assert code(f"idf_{fn}_attend", a) == -2
            a.workspace, a.workspace_bytes = AT + 16, nb.value
            assert code(f"idf_{fn}_attend", a) == -1


def test_python_refuses_what_does_not_fit():
    x = torch.zeros(4, 2, 16)
    with pytest.raises(ValueError):                                    # not on a GPU
        idf.norm_rotate(x, x, torch.zeros(4, dtype=torch.int64), torch.zeros(8, dtype=torch.float64))
    with pytest.raises(ValueError):
        idf.norm_rotate(x, x, torch.zeros(4, dtype=torch.int64), torch.zeros(8, dtype=torch.float64), layout="other")
    with pytest.raises(ValueError):
        idf.window_attend(x, x, x, window=4)
    with pytest.raises(ValueError):
        idf.decay_attend(x, x, x, torch.zeros(2))
    with pytest.raises(ValueError):
        idf.rotary_frequencies(64, scaling="other")


def test_rotary_frequencies():
    i = np.arange(32)
    plain = 10000.0 ** (-2.0 * i / 64)
    f, a = idf.rotary_frequencies(64)
    assert a == 1 and np.allclose(f.numpy(), plain, rtol=1e-14)
    f, a = idf.rotary_frequencies(64, scaling="linear", factor=4)
    assert a == 1 and np.allclose(f.numpy(), plain / 4, rtol=1e-14)
    f, a = idf.rotary_frequencies(64, scaling="base", factor=4)
    assert np.allclose(f.numpy(), (10000.0 * 4 ** (64 / 62)) ** (-2.0 * i / 64), rtol=1e-13)
    assert math.isclose(f[-1].item(), plain[-1] / 4, rel_tol=1e-12)     # the slowest pair as if divided by the factor
    f, a = idf.rotary_frequencies(64, scaling="parts", factor=8, trained=4096, fast=32, slow=1)
    turns = plain * 4096 / (2 * math.pi)
    assert math.isclose(a, 0.1 * math.log(8) + 1)
    got = f.numpy()
    assert np.allclose(got[turns >= 32], plain[turns >= 32]) and np.allclose(got[turns <= 1], plain[turns <= 1] / 8)
    between = (turns > 1) & (turns < 32)
    assert between.any() and np.all(got[between] < plain[between]) and np.all(got[between] > plain[between] / 8)
    for kw in (dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=258), dict(rotary_dim=64, base=1.0), dict(rotary_dim=64, scaling="linear", factor=0.5),
               dict(rotary_dim=2, scaling="base", factor=2), dict(rotary_dim=64, scaling="parts", factor=2, fast=1, slow=1), dict(rotary_dim=64, base=NAN)):
        with pytest.raises(idf.IdfError) as e:
            idf.rotary_frequencies(**kw)
        assert e.value.code == binding.IDF_EINVAL


# ---- the oracle against worked values and other forms ----

def test_oracle_rotation():
    y, _ = oracle.norm_rotate(np.array([[[1.0, 0.0, 5.0]]]), [1], [math.pi / 2], True, 2.0, None, 0.0)
    assert np.allclose(y, [[[0.0, 2.0, 5.0]]])                          # a quarter turn, twice as long
    y, _ = oracle.norm_rotate(np.array([[[3.0, 4.0, 0.0, 0.0]]]), [0], [1.0], False, 1.0, np.array([1.0, 2.0, 1.0, 1.0]), 0.0)
    assert np.allclose(y, [[[3 / 2.5, 8 / 2.5, 0, 0]]])                 # root of the mean of squares: 2.5
    # turning by p then q is turning by p + q
    x = np.random.default_rng(0).normal(size=(1, 2, 8))
    f = [1.0, 0.3, 0.01, 0.002]
    one, _ = oracle.norm_rotate(x, [1000], f, False, 1.0, None, 0)
    two, _ = oracle.norm_rotate(one, [77], f, False, 1.0, None, 0)
    assert np.allclose(two, oracle.norm_rotate(x, [1077], f, False, 1.0, None, 0)[0])


def test_oracle_attention():
    assert oracle.visible(5, 2, 1) == [0, 4, 5] and oracle.visible(1, 9, 3) == [0, 1] and oracle.visible(3, 1, 0) == [3]
    rng = np.random.default_rng(1)
    q, k, v = (rng.normal(size=(20, h, 4)) for h in (2, 1, 1))
    out, _, _ = oracle.Attention(6, 2, 0.5).push(q, k, v)
    mask = np.array([[j in oracle.visible(p, 6, 2) for j in range(20)] for p in range(20)])
    s = torch.from_numpy(0.5 * np.einsum("phd,jd->hpj", q, k[:, 0])).masked_fill(~torch.from_numpy(mask), -math.inf)
    assert np.allclose(out, np.einsum("hpj,jd->phd", torch.softmax(s, -1).numpy(), v[:, 0]))
    a = oracle.Attention(6, 2, 0.5)                                     # cut anywhere: the same
    assert np.allclose(out, np.concatenate([a.push(*(x[i:j] for x in (q, k, v)))[0] for i, j in ((0, 3), (3, 4), (4, 20))]))


def test_oracle_decay():
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(9, 2, 3)), rng.normal(size=(9, 1, 3)), rng.normal(size=(9, 1, 5))
    s0 = rng.normal(size=(1, 3, 5))
    out, _, end, _ = oracle.decay(q, k, v, [-0.3], s0, 0.7)
    lam = np.exp(-0.3 * (np.arange(9)[:, None] - np.arange(9)[None, :])) * np.tri(9)
    want = np.einsum("thd,jd,tj,je->the", q, k[:, 0], lam, v[:, 0]) + np.einsum("thd,de,t->the", q, s0[0], np.exp(-0.3 * np.arange(1, 10)))
    assert np.allclose(out, 0.7 * want)
    assert np.allclose(end[0], np.exp(-2.7) * s0[0] + np.einsum("j,jd,je->de", np.exp(-0.3 * np.arange(8, -1, -1)), k[:, 0], v[:, 0]))


def test_extension_names_do_not_depend_on_the_thread_that_asks(monkeypatch):
    """Threads of a build that ask for the interpreter's configuration while another reads it get None: names come from what was read at import."""
    import sysconfig

    from paper_1804_10727_amd import build
    want = sysconfig.get_config_var("EXT_SUFFIX")
    monkeypatch.setattr(sysconfig, "get_config_var", lambda name: None)
    assert want and build.push_path().endswith(want) and build.tokens_path().endswith(want)


def test_calls_of_many_parts_need_their_workspace():
    L = idf.load_library()
    for fn, a in (("window", window_args(heads_q=1, precision=1, head_dim=16, n_tokens=1, max_tokens=1, window=1 << 20, slots=1 << 20)),
                  ("decay", decay_args(heads_q=1, precision=1, n_tokens=1 << 20, max_tokens=1 << 20))):
        nb = C.c_size_t()
        assert getattr(L, f"idf_{fn}_workspace")(C.byref(a), C.byref(nb)) == 0 and nb.value > 0
        for at, size, want in ((None, 0, -2), (None, nb.value, -2), (AT, nb.value - 1, -2), (AT + 16, nb.value, -1)):
            a.workspace, a.workspace_bytes = at, size
            assert code(f"idf_{fn}_attend", a) == want, (fn, at, size)
