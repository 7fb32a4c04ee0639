"""Whether a result shares places with what is read, of other widths, types and numbers of rows, against the set of all their bytes."""
import random

import torch

from paper_1804_10727_amd import tokens


def places(t):
    size = t.element_size()
    return {t.data_ptr() + size * (r * (t.stride(0) if t.dim() == 2 else 0) + c) + i for r in range(t.shape[0] if t.dim() == 2 else 1) for c in range(t.shape[-1]) for i in range(size)}


def test_matrices_of_other_sizes():
    rng, seen = random.Random(5), set()
    buf = torch.zeros(1600, dtype=torch.int8)
    for _ in range(6000):
        row = rng.choice([40, 80, 120])            # bytes from row to row of the larger matrix
        pair = []
        for _ in range(2):
            dtype = rng.choice([torch.int8, torch.bfloat16, torch.float32])
            size = torch.empty(0, dtype=dtype).element_size()
            flat = buf.view(dtype)
            if rng.random() < 0.2:
                at = rng.randrange(0, 600 // size)
                pair.append(flat[at:at + rng.choice([1, 5, 30])])
                continue
            rows, cols, stride = rng.choice([1, 2, 3, 5]), rng.randrange(1, 40 // size + 1), rng.choice([row, row, row, 160]) // size
            pair.append(flat.as_strided((rows, cols), (stride, 1), rng.randrange(0, 640 // size)))
        a, b = pair
        want = bool(places(a) & places(b))
        got = tokens._share(a, b)
        alike = all(t.dim() == 1 or t.shape[0] == 1 for t in pair) or len({t.stride(0) * t.element_size() for t in pair if t.dim() == 2 and t.shape[0] > 1}) == 1
        wide = max(t.shape[-1] * t.element_size() for t in pair)
        tight = alike and (all(t.dim() == 1 or t.shape[0] == 1 for t in pair) or wide <= max(t.stride(0) * t.element_size() for t in pair if t.dim() == 2 and t.shape[0] > 1))
        assert got == want if tight else got >= want, (a.shape, a.stride(), a.dtype, b.shape, b.stride(), b.dtype, b.data_ptr() - a.data_ptr())
        assert got == tokens._share(b, a)
        seen.add((tight, got, want))
    assert {(True, True, True), (True, False, False)} <= seen
