"""The paged cache's state on the GPU: bad lengths and offsets, and compactions of many (slot,
head) pairs, bit for bit against the plain host model."""
import numpy as np
import pytest
import torch

from paper_2606_03928_amd import pages
from tests import page_model as pm
from tests.test_gpu_pages import BF16, F32, cumulative, ints, make, model, model_write, new_rows, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("length", [-1, -2 ** 31, 64 + 3, 2 ** 31 - 1])
def test_write_of_a_slot_whose_length_is_out_of_range(gpu_lib, length):
    # a table of 64 rows that are all there: of a length of 67 the last 5 tokens' rows are 62 .. 66
    c = make([64, 64, 20], 2, 16, 64, M=4, seed=90)
    c.length[1] = length
    m = model(c)
    kn, vn = new_rows(8, 2, 64, BF16, 91)
    c.write(kn, vn, ints([0, 1, 6, 8]))
    assert model_write(m, kn, vn, [0, 1, 6, 8]) == pm.BAD
    same(c, m, pages.STATUS_PAGE_BAD)
