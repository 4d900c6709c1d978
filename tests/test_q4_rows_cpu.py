"""Q4Cache.dense_rows: the struct holds an address, so the tensor behind it has to live as long."""
import gc
import weakref

import pytest
import torch

from paper_2609_03515_gb300 import Q4Cache


def test_packed_rows_keep_their_row_numbers():
    c = Q4Cache(2, 1, 2, 2, 64, 64, device="cpu", page_size=16)
    row0 = torch.tensor([0, 5], dtype=torch.int32)
    rows, alive = c.dense_rows(torch.zeros(1, 9, 2, 64), row0), weakref.ref(row0)
    assert rows.row0 == row0.data_ptr()
    del row0
    gc.collect()
    assert alive() is not None
    del rows
    gc.collect()
    assert alive() is None


@pytest.mark.parametrize("bad", [torch.tensor([0, 5]), torch.tensor([[0, 5], [1, 2]], dtype=torch.int32)[:, 0],
                                 torch.tensor([0], dtype=torch.int32)])
def test_row_numbers_of_another_kind_are_refused(bad):
    c = Q4Cache(2, 1, 2, 2, 64, 64, device="cpu", page_size=16)
    with pytest.raises(ValueError):
        c.dense_rows(torch.zeros(1, 9, 2, 64), bad)


def test_one_number_more_is_taken():
    """First rows of all sequences and the end of the last, as packed prompts often come with."""
    c = Q4Cache(2, 1, 2, 2, 64, 64, device="cpu", page_size=16)
    row0 = torch.tensor([0, 5, 9], dtype=torch.int32)
    assert c.dense_rows(torch.zeros(1, 9, 2, 64), row0).row0 == row0.data_ptr()
