"""Pages of the cache and beam search (include/earlytom_pages.h) where numbers, counts and orders are unlucky: against the plain
implementations of test_gpu_pages.py, with buffers between guards."""
import numpy as np
import pytest

from tests.test_gpu_decode import i32
from tests.test_gpu_pages import B, random_state, update_reference                                # noqa: F401

pytestmark = pytest.mark.gpu

GUARD = 4096


def guarded(values):
    """(the whole buffer, the part that holds `values`): int32 on the GPU between guards of -77."""
    v = np.asarray(values)
    wide = i32(np.full(v.size + 2 * GUARD, -77))
    part = wide[GUARD:GUARD + v.size].view(v.shape)
    part.copy_(i32(v))
    return wide, part


def guards_hold(wide):
    return bool((wide[:GUARD] == -77).all()) and bool((wide[-GUARD:] == -77).all())


# ---- et_pages_update --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n_seq,longest,rows", [(5, 144, 0), (40, 100, 100), (40, 100, 33_000), (700, 900, 50), (1500, 900, 40_000), (9000, 40, 64),
                                                (20_000, 70, 33_000)])
def test_update_of_sums_beyond_32_bits_leaves_tables_right(B, n_seq, longest, rows):              # noqa: F811
    """Many sequences ask for nearly 2^31 positions each: none of them gets one, and tables, counts and lengths are what they are without
    them.  Full sequences among them, the last one too, whose entries end where the next row or the buffer's end is."""
    rng = np.random.default_rng(n_seq + rows)
    page = 16
    lens, table, refs = random_state(rng, n_seq, longest, page, 4000, room=0)
    cap = table.shape[1] * page
    full = rng.random(n_seq) < 0.3
    full[-1] = full[n_seq // 2] = True
    keep = np.where(full, cap, np.maximum(lens - 3, -1))
    lens = np.where(full, cap, lens)
    table[full] = rng.integers(0, len(refs), (int(full.sum()), table.shape[1]))
    refs = np.maximum(refs, 0) + np.bincount(table[full].ravel(), minlength=len(refs))
    add = np.where(rng.random(n_seq) < 0.6, 2 ** 31 - 1 - rng.integers(0, 9, n_seq), rng.integers(0, 9, n_seq))
    want = update_reference(refs, page, table, lens, keep, add.astype(object), most=0)
    bufs = [guarded(x) for x in (refs, table, np.full(n_seq, -9), np.full(n_seq + 1, -9), np.full(max(rows, 1), -9))]
    status = i32([0])
    B.et_pages_update(bufs[0][1], page, bufs[1][1], i32(lens), i32(keep), i32(add), bufs[2][1], bufs[3][1], bufs[4][1] if rows else None, status)
    assert all(guards_hold(wide) for wide, _ in bufs)
    for (_, got), expected in zip(bufs, want[:3]):
        assert np.array_equal(got.cpu().numpy(), expected)
    assert status.item() >= max(want[5])                  # (rows of no order may meet entries that are no pages)
