"""What calls of the operators that mix tokens launch, on a stand-in for the HIP runtime (no GPU): the plan of a launch and the workspace that was
asked for are one plan."""
import pytest

import host_runtime

AT = 1 << 40                 # addresses that nobody reads


@pytest.fixture(scope="session")
def runtime(tmp_path_factory):
    return host_runtime.build(tmp_path_factory.mktemp("runtime"))


def decay_args(precision, max_tokens, n_tokens, segments=2, heads=2, dim_k=64, dim_v=64, workspace=None, workspace_bytes=0):
    from paper_1804_10727_amd import tokens
    q, v = tokens._Tokens(AT, heads * dim_k, dim_k), tokens._Tokens(AT, heads * dim_v, dim_v)
    return tokens._Decay(precision, heads, heads, dim_k, dim_v, n_tokens, max_tokens, segments, segments, 0.125, q, q, v, v, AT, AT, AT, AT, None,
                         workspace, workspace_bytes)


def attend(rt, a):
    import ctypes as C

    from paper_1804_10727_amd import binding
    rt.host_begin()
    rc = binding.load_library().idf_decay_attend(C.byref(a), None)
    assert rt.host_error() == b"", rt.host_error()
    return rc


def workspace(a):
    import ctypes as C

    from paper_1804_10727_amd import binding
    nb = C.c_size_t(1 << 60)
    assert binding.load_library().idf_decay_workspace(C.byref(a), C.byref(nb)) == 0
    return nb.value


def decay_without_tokens(rt):
    for precision in (0, 1):
        for max_tokens in (0, 1, 64, 128, 256, 1024, 4096, 1 << 20):
            for dim_k in (32, 64, 128, 256):
                a = decay_args(precision, max_tokens, 0, dim_k=dim_k)
                assert workspace(a) == 0 and attend(rt, a) == 0
                # the states are handed on, by one kernel and in one part
                assert rt.host_launches(None) == 1 and rt.host_launches(b"k_decay_scan") == 0, (precision, max_tokens, dim_k)


def test_decay_without_tokens_needs_no_parts(runtime):
    """A bound on the tokens of a segment says nothing where no stream brings any."""
    host_runtime.run(runtime, "test_tokens_host", "decay_without_tokens")


def decay_plans(rt):
    seen = set()
    for precision in (0, 1):
        for segments in (1, 3, 64, 5000):
            for heads in (1, 16):
                for dim_k, dim_v in ((64, 64), (128, 200), (256, 32)):
                    for n_tokens in (0, 1, 5, 31, 32, 200, 5000, 300000):
                        for max_tokens in (0, 1, 2, 33, 127, 128, 256, 4096, 300000):
                            args = dict(precision=precision, max_tokens=max_tokens, n_tokens=n_tokens, segments=segments, heads=heads, dim_k=dim_k, dim_v=dim_v)
                            need = workspace(decay_args(**args))
                            seen.add(need > 0)
                            if need:
                                assert attend(rt, decay_args(**args)) == -2 and rt.host_launches(None) == 0, args
                                assert attend(rt, decay_args(**args, workspace=AT, workspace_bytes=need - 1)) == -2 and rt.host_launches(None) == 0, args
                            assert attend(rt, decay_args(**args, workspace=AT if need else None, workspace_bytes=need)) == 0, args
                            assert rt.host_launches(b"k_decay_scan") == (1 if need else 0), args
                            assert need % (heads * segments * dim_k * dim_v * 4) == 0
    assert seen == {False, True}


def test_decay_launches_parts_only_into_a_workspace(runtime):
    host_runtime.run(runtime, "test_tokens_host", "decay_plans")
