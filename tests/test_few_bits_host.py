"""What calls of the layers in few bits and of the gated recurrence launch, on a stand-in for the HIP runtime (no GPU): the plan of a launch and the workspace
that was asked for are one plan, and what a launch cannot take is refused before it."""
import ctypes as C

import pytest

import host_runtime

AT = 1 << 40                 # addresses that nobody reads


@pytest.fixture(scope="session")
def runtime(tmp_path_factory):
    return host_runtime.build(tmp_path_factory.mktemp("runtime"))


def call(rt, name, a):
    from paper_1804_10727_amd import binding
    rt.host_begin()
    rc = getattr(binding.load_library(), name)(C.byref(a), None)
    assert rt.host_error() == b"", rt.host_error()
    return rc


def workspace(name, a):
    from paper_1804_10727_amd import binding
    nb = C.c_size_t(1 << 60)
    assert getattr(binding.load_library(), name.replace("project_rows", "project") + "_workspace")(C.byref(a), C.byref(nb)) == 0, a
    return nb.value


def holds_its_plan(rt, name, make, args, launches):
    """The call of make(**args) takes exactly the workspace that was asked for, and launches nothing into less; launches(bytes): kernels and how often."""
    need = workspace(name, make(**args))
    if need:
        for kw in (dict(), dict(workspace=AT, workspace_bytes=need - 1)):
            assert call(rt, name, make(**args, **kw)) == -2 and rt.host_launches(None) == 0, args
        assert call(rt, name, make(**args, workspace=AT + 64, workspace_bytes=need)) == -1 and rt.host_launches(None) == 0, args
    assert call(rt, name, make(**args, workspace=AT if need else None, workspace_bytes=need)) == 0, args
    for kernel, n in launches(need).items():
        assert rt.host_launches(kernel) == n, (args, kernel, rt.host_launches(kernel))
    return need


def project_args(precision, out, cols, n_out, rows, workspace=None, workspace_bytes=0):
    from paper_1804_10727_amd import tokens
    return tokens._Project(precision, out, cols, n_out, rows, tokens._Rows(AT, (cols + 15) // 16 * 16), tokens._Rows(AT, n_out), AT if precision == 2 else None, AT, AT, None,
                           workspace, workspace_bytes)


def project_plans(rt):
    for precision in (0, 1, 2):
        for out in (0, 1):
            for rows in (0, 1, 16, 17, 200, 5000, (1 << 24) - 1):
                for cols, n_out in ((16, 1), (64, 8192), (4096, 6144), (65536, 100)):
                    need = holds_its_plan(rt, "idf_project_rows", project_args, dict(precision=precision, out=out, cols=cols, n_out=n_out, rows=rows),
                                          lambda need: {None: (rows > 0) + (need > 0), b"k_quantize_rows": need > 0, b"k_project_few": 0 < rows <= 16, b"k_project_tile": rows > 16})
                    assert need == (0 if precision == 2 else rows * (cols + 4))


def window_args(rows, max_tokens, heads, kv, dim, precision, segments, window, workspace=None, workspace_bytes=0):
    from paper_1804_10727_amd import tokens
    q = tokens._Tokens(AT, heads * dim, dim)
    slots = 4 + window + min(rows, max_tokens)
    return tokens._NibbleAttend(precision, heads, kv, dim, rows, max_tokens, segments, segments, slots, window, 4, 0.125, q, q, tokens._NibbleRing(AT, AT, AT, AT), AT, AT, AT,
                                workspace, workspace_bytes)


def attend_plans(rt):
    seen = set()
    for precision in (0, 1):
        for segments in (1, 3, 64, 5000):
            for heads, kv in ((1, 1), (32, 4), (24, 1)):
                for dim in (32, 96, 128, 256):
                    for rows in (0, 1, 64, 5000):
                        for max_tokens in (0, 1, 5, 4096):
                            for window in (1, 100, 40000):
                                need = holds_its_plan(rt, "idf_nibble_attend", window_args, dict(rows=rows, max_tokens=max_tokens, heads=heads, kv=kv, dim=dim, precision=precision, segments=segments, window=window),
                                                      lambda need: {None: (rows > 0 and max_tokens > 0) + (need > 0), b"k_window_join": need > 0})
                                assert need % (rows * heads * (dim + 2) * 4 or 1) == 0
                                seen.add((need > 0, bool(rt.host_launches(b"k_nibble_step")), bool(rt.host_launches(b"k_nibble_tile"))))
    assert seen == {(False, False, False), (False, True, False), (False, False, True), (True, True, False), (True, False, True)}


def gate_args(rows, max_tokens, channels, precision, segments, back=False, workspace=None, workspace_bytes=0):
    from paper_1804_10727_amd import tokens
    r = tokens._Rows(AT, channels)
    if back:
        return tokens._GateScanBackward(precision, channels, rows, max_tokens, segments, segments, r, r, r, r, r, AT, AT, AT, AT, None, workspace, workspace_bytes)
    return tokens._GateScan(precision, channels, rows, max_tokens, segments, segments, r, r, r, AT, AT, AT, AT, None, workspace, workspace_bytes)


def gate_plans(rt):
    seen = set()
    for back in (False, True):
        for precision in (0, 1):
            for segments in (1, 3, 64, 5000):
                for channels in (1, 100, 2048):
                    for rows in (0, 1, 17, 300, 5000, 300000):
                        for max_tokens in (0, 1, 15, 17, 4096, 1 << 20):
                            need = holds_its_plan(rt, "idf_gate_scan_backward" if back else "idf_gate_scan", lambda **kw: gate_args(**kw, back=back),
                                                  dict(rows=rows, max_tokens=max_tokens, channels=channels, precision=precision, segments=segments),
                                                  lambda need: {None: 1 + (need > 0), b"k_gate_absent": need > 0, b"k_gate_back_tile" if back else b"k_gate_tile": 1})
                            seen.add(need > 0)
                            # one launch for segments of one tile; twelve bytes a channel for every 128 tokens and every segment are enough
                            assert (need > 0) == (min(rows, max_tokens) > (128 if back else 256)) and need <= (rows // 128 + segments + 1) * channels * 12 + 256 + 16
    assert seen == {False, True}


@pytest.mark.parametrize("plans", ["project_plans", "attend_plans", "gate_plans"])
def test_launches_go_by_the_workspace_that_was_asked_for(runtime, plans):
    host_runtime.run(runtime, "test_few_bits_host", plans)


def more_than_a_launch_takes(rt):
    from paper_1804_10727_amd import tokens
    for rows, n_out, rc in ((1 << 23, 1 << 14, 0), ((1 << 24) - 1, 1 << 14, -5), (1 << 14, 1 << 24, -5), (1 << 13, 1 << 24, 0), (17, 1 << 24, 0), ((1 << 24) - 1, 1, 0)):
        a = project_args(2, 1, 64, n_out, rows)
        assert call(rt, "idf_project_rows", a) == rc, (rows, n_out)
        assert rt.host_launches(None) == (rc == 0)
    for n, rc in ((1 << 26, 0), ((1 << 26) + 1, -5)):
        t = tokens._Tokens(AT, 32, 32)
        a = tokens._NibbleAppend(1, 1, 32, 32, 0, n, (1 << 31) - 1, 1, 1, 64, 2, 1.0, 1e-6, t, t, tokens._NibbleRing(AT, AT, AT, AT), AT, None, AT, AT, None)
        assert call(rt, "idf_nibble_append", a) == rc and rt.host_launches(None) == (rc == 0)
    for rows, channels, rc in ((1 << 29, 1 << 6, 0), (1 << 30, 1 << 8, -5), ((1 << 31) - 1, 65, -5), (1 << 18, 1 << 16, 0), (1 << 18, 1 << 20, -5)):
        for back in (False, True):
            a = gate_args(rows, 4096, channels, 0, 1000, back, AT, 1 << 50)
            a.offsets = AT
            assert call(rt, "idf_gate_scan_backward" if back else "idf_gate_scan", a) == rc and (rt.host_launches(None) > 0) == (rc == 0), (rows, channels, back)
    # heads of many streams go in several launches
    for streams, heads, launches in ((1, 1, 1), (64, 1000, 1), (65, 1000, 2), (200000, 1, 4)):
        a = tokens._NibbleValues(1, heads, 32, streams, 5, tokens._NibbleRing(AT, AT, AT, AT), AT, AT)
        assert call(rt, "idf_nibble_values", a) == 0 and rt.host_launches(b"k_nibble_values") == launches


def test_calls_beyond_a_launch(runtime):
    host_runtime.run(runtime, "test_few_bits_host", "more_than_a_launch_takes")
