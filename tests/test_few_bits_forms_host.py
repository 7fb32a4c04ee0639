"""Which form of a kernel the calls of test_gpu_few_bits_forms.py take, on a stand-in for the HIP runtime (no GPU): a rule that is measured anew does not leave a form
untested without a word."""
import pytest

import host_runtime
from test_few_bits_host import AT, call, gate_args, project_args, workspace

# name of the tile, stages on their way, and (rows, outputs) that go in it: with remainders, whole lines and single values
TILES = {"64x32": ("Li2ELi2ELi2ELi1ELi6ELi2E", 6, ((17, 33), (64, 160), (100, 1000))), "64x64": ("Li2ELi2ELi2ELi2ELi4ELi2E", 4, ((17, 8193), (50, 16000))),
         "64x128": ("Li2ELi2ELi2ELi4ELi3ELi2E", 3, ((91, 8193), (128, 12800))), "128x128": ("Li2ELi2ELi4ELi4ELi2ELi2E", 2, ((461, 8193), (512, 8320))),
         "256x256": ("Li4ELi2ELi4ELi8ELi2ELi1E", 2, ((979, 8193), (1024, 8208)))}
# streams, query heads, key/value heads, head size, window, first tokens, tokens of a segment at most, and rows, in tiles of 16, of a workgroup of the attention's kernel for few rows, by float32 and bfloat16
STEPS = [(40, 16, 8, 64, 600, 3, 1, (1, 1)), (40, 32, 8, 128, 300, 5, 1, (1, 1)), (40, 8, 8, 96, 200, 0, 20, (2, 2)), (40, 16, 8, 32, 130, 7, 12, (2, 2)), (40, 16, 8, 128, 100, 2, 16, (2, 2)),
         (40, 8, 8, 256, 150, 1, 5, (1, 1)), (40, 8, 8, 160, 70, 0, 16, (1, 1)), (40, 128, 8, 64, 40, 2, 2, (2, 2)), (20, 8, 8, 64, 3000, 4, 1, (1, 1)), (33, 24, 8, 128, 700, 0, 9, (2, 2))]
# lengths, channels and, by float32, bfloat16, the values of a lane of the recurrence's forward pass in a chain of tiles with 32 tokens to a wave
CHAINS = [((4097, 255, 4095, 257), 2048, (1, 2)), ((8192 + 31, 1, 0, 700), 1023, (1, 1)), ((4096, 4096, 33), 1902, (1, 2))]


@pytest.fixture(scope="session")
def runtime(tmp_path_factory):
    return host_runtime.build(tmp_path_factory.mktemp("runtime"))


def tiles(rt):
    for which, (name, _, shapes) in TILES.items():
        for rows, outs in shapes:
            for out in (0, 1):
                for cols in (16, 500, 2000):
                    assert call(rt, "idf_project_rows", project_args(2, out, -(-cols // 16) * 16, outs, rows)) == 0
                    assert rt.host_launches(f"k_project_tileI{'DF16b' if out else 'f'}{name}".encode()) == 1, (which, rows, outs)


def steps(rt):
    from paper_1804_10727_amd import tokens
    for streams, hq, hkv, dim, window, sinks, longest, tall in STEPS:
        for precision in (0, 1):
            n = streams * longest
            q = tokens._Tokens(AT, hq * dim, dim)
            a = tokens._NibbleAttend(precision, hq, hkv, dim, n, longest, streams, streams, sinks + window + longest, window, sinks, 0.125, q, q, tokens._NibbleRing(AT, AT, AT, AT), AT, AT, None, None, 0)
            a.workspace, a.workspace_bytes = AT, workspace("idf_nibble_attend", a)
            assert call(rt, "idf_nibble_attend", a) == 0
            padded = 64 if dim <= 64 else 128 if dim <= 128 else 256
            assert rt.host_launches(f"k_nibble_stepILi{precision}ELi{padded}ELi{tall[precision]}ELi4EE".encode()) == 1, (streams, hq, hkv, dim, precision)
            assert (rt.host_launches(b"k_window_join") > 0) == (window == 3000)


def chains(rt):
    for lengths, channels, values in CHAINS:
        for precision in (0, 1):
            a = gate_args(sum(lengths), max(lengths), channels, precision, len(lengths))
            a.offsets = AT
            a.workspace, a.workspace_bytes = AT, workspace("idf_gate_scan", a)
            assert call(rt, "idf_gate_scan", a) == 0
            assert rt.host_launches(f"k_gate_tileILi{precision}ELi{values[precision]}ELi2ELb1EE".encode()) == 1, (lengths, channels, precision)


@pytest.mark.parametrize("forms", ["tiles", "steps", "chains"])
def test_forms(runtime, forms):
    host_runtime.run(runtime, "test_few_bits_forms_host", forms)
