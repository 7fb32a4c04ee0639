"""project_rows into a result that the caller gives: refused where it shares places with what is read, taken where it lies beside it."""
import pytest
import torch

import paper_1804_10727_amd as idf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("rows", [1, 5, 300])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_out_over_what_is_read(rows, dtype):
    g = torch.Generator().manual_seed(rows)
    both = torch.randn(rows, 256, generator=g).to(dtype).to(DEV)
    w, ws = idf.quantize_rows(torch.randn(64, 96, generator=g).to(DEV))
    bias = torch.randn(64, generator=g).to(DEV)
    x = both[:, :96]
    want = idf.project_rows(x, w, ws, bias=bias)
    was = both.clone()
    for bad in (both[:, :64], both[:, 32:96], both[:, 95:159], both.flatten()[:rows * 64].view(rows, 64)):
        with pytest.raises(ValueError, match="shares"):
            idf.project_rows(x, w, ws, bias=bias, out=bad)
    assert torch.equal(both, was)
    for at in (96, 101, 192):
        out = both[:, at:at + 64]
        assert idf.project_rows(x, w, ws, bias=bias, out=out) is out and torch.equal(out, want)
        assert torch.equal(both[:, :96], was[:, :96])
    codes, scales = idf.quantize_rows(x)
    kept = codes.clone()
    over = codes.view(dtype)                       # [rows][96 / size]
    narrow, narrow_s = w[:over.shape[1]].contiguous(), ws[:over.shape[1]].contiguous()
    with pytest.raises(ValueError, match="shares"):
        idf.project_rows(codes, narrow, narrow_s, x_scales=scales, out=over)
    assert torch.equal(codes, kept)
    if dtype == torch.float32:
        one = torch.zeros(64, device=DEV)
        for kw in (dict(weight_scales=one), dict(weight_scales=ws, bias=one)):
            with pytest.raises(ValueError, match="shares"):
                idf.project_rows(x[:1], w, **kw, out=one[None])
        with pytest.raises(ValueError, match="shares"):
            idf.project_rows(x[:1], w, ws, out=w.view(torch.float32).flatten()[:64][None])


def test_codes_that_the_caller_gives_beside_a_result():
    """Codes, scales and a result that lie behind each other in one piece of memory."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(48, 64, generator=g).to(DEV)
    w, ws = idf.quantize_rows(torch.randn(32, 64, generator=g).to(DEV))
    want = idf.project_rows(x, w, ws)
    memory = torch.zeros(48 * 64 + 48 * 4 + 48 * 32 * 4, dtype=torch.int8, device=DEV)
    codes, scales, out = memory[:48 * 64].view(48, 64), memory[48 * 64:48 * 68].view(torch.float32), memory[48 * 68:].view(torch.float32).view(48, 32)
    idf.quantize_rows(x, codes=codes, scales=scales)
    assert torch.equal(idf.project_rows(codes, w, ws, x_scales=scales, out=out), want)
