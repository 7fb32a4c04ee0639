"""What calls of the gated recurrence launch where there is little or nothing to go over, on a stand-in for the HIP runtime (no GPU)."""
import pytest

import host_runtime
from test_few_bits_host import AT, call, gate_args, workspace


@pytest.fixture(scope="session")
def runtime(tmp_path_factory):
    return host_runtime.build(tmp_path_factory.mktemp("runtime"))


def rows_of_no_segment(rt):
    """The backward pass sets them to zero where there are no segments at all, too: one launch, no workspace, whatever max_tokens says."""
    for precision in (0, 1):
        for rows, max_tokens in ((100, 100), (100, 0), (300000, 1 << 20)):
            a = gate_args(rows, max_tokens, 64, precision, 0, back=True)
            a.offsets = AT
            assert workspace("idf_gate_scan_backward", a) == 0
            assert call(rt, "idf_gate_scan_backward", a) == 0 and rt.host_launches(None) == rt.host_launches(b"k_gate_back_tile") == 1
            a.grad_gates.base = None
            assert call(rt, "idf_gate_scan_backward", a) == -1 and rt.host_launches(None) == 0
    a = gate_args(0, 0, 64, 0, 0, back=True)
    a.offsets = AT
    assert call(rt, "idf_gate_scan_backward", a) == 0 and rt.host_launches(None) == 0


def rows_to_clear(rt):
    """The forward pass does where it is asked to, in the launch that it has anyway."""
    for precision in (0, 1):
        for segments, rows, max_tokens in ((0, 100, 100), (0, 300000, 1 << 20), (3, 5000, 0), (3, 5000, 1), (3, 5000, 200), (3, 300000, 4096)):
            for clear in (0, 1):
                a = gate_args(rows, max_tokens, 64, precision, segments)
                a.offsets, a.clear_rows, a.state_out = AT, clear, None
                a.workspace, a.workspace_bytes = AT, workspace("idf_gate_scan", a)
                assert call(rt, "idf_gate_scan", a) == 0
                assert rt.host_launches(b"k_gate_tile") == (clear or (segments > 0 and max_tokens > 0)) and rt.host_launches(None) - rt.host_launches(b"k_gate_absent") <= 1
                a.out.base = None
                assert call(rt, "idf_gate_scan", a) == (-1 if clear or (segments and max_tokens) else 0) and rt.host_launches(None) == 0


def test_rows_to_clear(runtime):
    host_runtime.run(runtime, "test_gate_scan_host", "rows_to_clear")


def test_rows_of_no_segment(runtime):
    host_runtime.run(runtime, "test_gate_scan_host", "rows_of_no_segment")
