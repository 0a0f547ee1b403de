"""The paged cache's state on the GPU: bad lengths and offsets, and compactions of many (slot,
head) pairs, bit for bit against the plain host model."""
import ctypes

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


def test_write_of_offsets_that_fall_stays_within_the_rows(gpu_lib):
    # the search for token 5 ends at slot 2, whose tokens the offsets say are 1 .. 2
    c = make([9, 9, 9, 9], 2, 16, 64, garbage=5.0, seed=92)
    kn, vn = new_rows(10, 2, 64, BF16, 93)
    c.write(kn, vn, ints([0, 9, 1, 2, 30]))
    torch.cuda.synchronize()
    for s in range(4):
        for x in (c.k, c.v):
            assert (x[int(c.table[s, 0]), :, 9:] == 5).all()
    assert int(c.status) == pages.STATUS_PAGE_BAD


def test_workspace_sizes_refuse_floats(gpu_lib):
    c = make([3000, 900], 1, 16, 64, seed=94)
    for again in range(2):
        assert c.attn_workspace_bytes(2, 2, 1) > 0
        q = new_rows(2, 2, 64, BF16, 95)[0]
        c.attn(q, ints([0, 1, 2]), 1)
        for sizes in ((2, 2, 1.0), (2.0, 2, 1), (2, 2.0, 1), (2, 2, 1, 3000.0)):
            with pytest.raises(ctypes.ArgumentError):
                c.attn_workspace_bytes(*sizes)
        with pytest.raises(ctypes.ArgumentError):
            c.attn(q, ints([0, 1, 2]), 1.0)
