"""The largest page tables: slots that CTAs look at behind a sequence's end have numbers of 32 bits."""
import pytest

import torch

from paper_2504_14051_b200 import binding as C

MOST = (1 << 31) - (1 << 16)


def workspace(page_size, max_pages, dtype=torch.float32):
    return C.caote_paged_workspace_bytes(C.make_paged_params(1, 2, 1, 64, page_size, 8, max_pages, 1, 1, dtype, 0.1))


@pytest.mark.parametrize("page_size", [16, 32, 64, 128, 256])
def test_slots_of_a_sequence(page_size):
    assert workspace(page_size, MOST // page_size) > 0
    assert workspace(page_size, MOST // page_size + 1) == 0
    assert workspace(page_size, (1 << 31) // page_size - 1) == 0
