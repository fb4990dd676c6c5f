"""fa_tree_words of masks that are not of type bool: what is not zero is seen."""
import pytest
import torch

from paper_2407_08608_amd import binding


@pytest.mark.parametrize("dtype,one", [(torch.uint8, 255), (torch.int8, -1), (torch.int32, 6), (torch.int64, 1 << 40), (torch.float32, 0.5), (torch.bool, True)])
def test_any_type_of_mask(dtype, one):
    seen = torch.rand((2, 40, 40), generator=torch.Generator().manual_seed(1)) < 0.3
    words = binding.fa_tree_words(torch.where(seen, torch.tensor(one, dtype=dtype), torch.tensor(0, dtype=dtype)))
    assert torch.equal(words, binding.fa_tree_words(seen))
