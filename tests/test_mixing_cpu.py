"""What the mixer of a net's rows refuses before anything is worked on: host code, no GPU needed."""
import pytest
import torch

from paper_1804_10727_amd.mixing import TokenMixer


@pytest.mark.parametrize("rows,counts", [(4, None), (5, None), (6, (1, 2, 2)), (6, (3, 3, 3)), (0, (1, 0, 0)), (6, (2, 4)), (6, (2, 2, 1, 1)), (6, (7, 0, -1)),
                                         (6, torch.tensor([2, 2, 3])), (3, (1, 1, 0.5))])
def test_numbers_of_rows_that_do_not_add_up(rows, counts):
    """Positions are laid out by the counts: too many would be written past the rows' end."""
    m = TokenMixer(16, 3, heads=2, kv_heads=1, dim=16, window=8, device="cpu")
    with pytest.raises(ValueError, match="rows"):
        m.push(torch.zeros(rows, 16), counts)
    assert m.starts.tolist() == [0, 0, 0]
