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


def test_offsets_are_checked_before_ids_are_read():
    """Offsets that rise past the table's end and fall back to it: refused before an id behind the end is looked at (there is
    no table here at all, which would be INVALID_ARG)."""
    off = np.array([0, 10, 5], np.int64)
    assert status(B.pdkv_seqs_create, pool(), [160, 0], off, None, num_q_heads=8, q_tokens=1) == B.PDKV_ERR_TABLE
    off, tbl = csr([40, 7], 16)
    assert status(B.pdkv_seqs_create, pool(), [40, 7], off, tbl, prefix_len=[160, 0], prefix_tbl_off=np.array([0, 10, 5], np.int64), prefix_tbl=None,
                  seq_prefix=[0, 1], num_q_heads=8, q_tokens=1) == B.PDKV_ERR_TABLE
