"""What a batch was made of cannot be exchanged afterwards: the structure that calls read would not follow."""
import pytest
import torch

from paper_2512_24449_amd import binding


def test_attributes_are_read_only():
    lens, table = torch.ones(2, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int32)
    made = binding.FP4Batch(lens, 5, table)
    assert (made.batch, made.max_new, made.table_pages, made.device) == (2, 5, 3, lens.device)
    for name, other in (("batch", 1), ("max_new", 7), ("table_pages", 2), ("device", "cuda:1"), ("lens", lens.clone()),
                        ("page_table", table.clone()), ("new_rows", lens), ("first_row", lens)):
        with pytest.raises(AttributeError):
            setattr(made, name, other)
    assert (made.max_new, made._c.max_new, made._c.batch, made._c.table_pages) == (5, 5, 2, 3) and made.lens is lens
