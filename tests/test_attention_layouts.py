"""How the attention helpers read the layout of one token's heads (no GPU)."""

import torch

from paper_2606_07116_gb300 import offq as Q


def test_the_way_to_the_next_token_does_not_matter_with_one():
    """A single token from a buffer whose rows are not a multiple of 16 bytes, or that overlap: heads are contiguous and
    there is no next row."""
    rows = torch.zeros((4, 3 * 128 + 4), dtype=torch.bfloat16)
    one = rows.as_strided((1, 3, 128), (388, 128, 1))
    assert Q._heads(one) == (1, 3, 128, 384)
    assert Q._heads(torch.zeros(128).expand(1, 1, 128)) == (1, 1, 128, 128)
    assert Q._heads(rows.as_strided((4, 3, 128), (388, 128, 1))) == (4, 3, 128, 388)
