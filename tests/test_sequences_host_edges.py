"""Corners of the handles of cached sequences and of their calls without a GPU."""
import numpy as np
import pytest

from paper_2408_08147_b200 import binding as B
from test_sequences_host import FAKE, args, built, create, csr, pool, status  # noqa: F401 (`built` is a fixture)


def test_row_counts_past_32_and_64_bits():
    """q_tokens x num_q_heads x n_seq is limited whatever it would wrap to (2^31 - 1, 2^31 - 4 and 4: below zero)."""
    p = pool()
    for lens, Hq, Q in (([4] * 4, 2 ** 31 - 4, 2 ** 31 - 1), ([4] * 8, 2 ** 30, 2 ** 31 - 1), ([4], 2 ** 30, 2 ** 30),
                        ([4] * 3, 4, 1 << 27), ([], 4, (1 << 28) + 1)):
        assert status(create, p, lens, Hq=Hq, q_tokens=Q) == B.PDKV_ERR_INVALID_ARG
