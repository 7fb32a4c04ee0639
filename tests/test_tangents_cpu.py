"""Tensors of torch's forward mode are refused before anything else is asked of them: a result without a tangent would stand for a derivative of zero."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_1804_10727_amd as idf


@pytest.mark.parametrize("call", [lambda x: idf.quantize_rows(x), lambda x: idf.project_rows(x, x.to(torch.int8), x[0]), lambda x: idf.project_rows(x.detach(), x.to(torch.int8), x[0].detach(), bias=x[0]),
                                  lambda x: idf.gate_scan(x, x), lambda x: idf.gate_scan(x.detach(), x.detach(), x[:1]), lambda x: idf.gate_scan_backward(x.detach(), x.detach(), x[0].detach(), x),
                                  lambda x: idf.nibble_attend(x[None], [x] * 4, window=4), lambda x: idf.nibble_append(x[None], x[None], [x] * 4),
                                  lambda x: idf.norm_rotate(x[None], x[None], x, x), lambda x: idf.window_attend(x[None], x[None], x[None], window=4), lambda x: idf.decay_attend(x[None], x[None], x[None], x[0])])
def test_tangents_are_refused(call):
    x = torch.zeros(4, 64)
    with forward_ad.dual_level():
        for dual in (forward_ad.make_dual(x, torch.ones(4, 64)), forward_ad.make_dual(torch.zeros(8, 64), torch.ones(8, 64))[4:]):
            for mode in (torch.enable_grad, torch.no_grad):
                with mode(), pytest.raises(ValueError, match="tangent"):
                    call(dual)
        with pytest.raises(ValueError) as e:
            call(x)
        assert "tangent" not in str(e.value)
