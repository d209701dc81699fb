"""Without a GPU: what a call on the cache asks for in memory, whatever its hints say."""

import ctypes

import numpy as np

from paper_2607_02893_amd import vbq

A = 1 << 20  # an address that nothing here looks at
MOST = 1 << 18  # VBQ_KV_MAX_PARTS


def _workspace(heads, D, group, **kw):
    d, n = vbq.VbqKvDesc(), ctypes.c_size_t(0)
    assert vbq.lib().vbq_kv_layout(1000, heads, D, ctypes.byref(d)) == 0
    f = dict(n_seqs=1, table_stride=2048, page_table=A, row_start=A, seq_len=A, n_rows=1, max_rows=1, max_len=131072)
    f.update(kw)
    b = vbq.VbqKvBatch(*[f[n] for n in ("n_seqs", "table_stride", "page_table", "row_start", "seq_len", "n_rows",
                                        "max_rows", "max_len")])
    assert vbq.lib().vbq_kv_attention_workspace_size(ctypes.byref(d), ctypes.byref(b), heads * group, ctypes.byref(n)) == 0
    return n.value


def test_a_workspace_is_bounded_whatever_the_hints():
    # a prompt whose rows are said to be one
    assert _workspace(8, 128, 4, n_rows=8192) <= MOST * 130 * 4
    rng = np.random.default_rng(1)
    for _ in range(20000):
        heads, D, group = int(2 ** rng.uniform(0, 10)), int(rng.choice([64, 128, 256])), int(2 ** rng.uniform(0, 8))
        n_rows = min(int(2 ** rng.uniform(0, 30)), (1 << 30) // group)
        n = _workspace(heads, D, group, n_seqs=int(2 ** rng.uniform(0, 16)), n_rows=n_rows,
                       max_rows=int(2 ** rng.uniform(0, 30)), max_len=int(2 ** rng.uniform(0, 31)))
        assert n <= MOST * (D + 2) * 4


def test_right_hints_stay_below_the_bound():
    """The bound binds nobody who says how many rows there are."""
    rng = np.random.default_rng(2)
    split = 0
    for _ in range(20000):
        heads, D, group = int(2 ** rng.uniform(0, 10)), int(rng.choice([64, 128, 256])), int(2 ** rng.uniform(0, 8))
        n_seqs = int(2 ** rng.uniform(0, 10))
        rows = max(1, min(int(2 ** rng.uniform(0, 14)), (1 << 30) // (group * n_seqs)))
        n = _workspace(heads, D, group, n_seqs=n_seqs, row_start=None, n_rows=n_seqs * rows, max_rows=rows,
                       max_len=int(2 ** rng.uniform(0, 31)))
        assert n <= 16 * 1536 * (D + 2) * 4
        split += n > 0
    assert split > 1000
