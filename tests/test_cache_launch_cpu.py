"""Without a GPU: what a call on the cache asks for in memory and workgroups, whatever its hints say."""

import ctypes
import os
import subprocess

import numpy as np

from paper_2607_02893_amd import vbq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
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


HOST = r"""
#include "paper_2607_02893_amd/csrc/vbq_cache.hpp"
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#define NEED(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); std::exit(1); } } while (0)
int main() {
  const int64_t counts[] = {1, 2, 31, 32, 33, 1000, 65535, 1 << 20, 1 << 30};
  for (int64_t max_rows : counts) for (int64_t n_rows : counts) for (int64_t heads : {1, 3, 8, 1024}) for (int64_t seqs : {1, 16, 1000, 65535}) {
    const int64_t n = vbq::blocks_of(max_rows, n_rows, heads, seqs), all = n * heads * seqs;
    const int64_t rows = max_rows < n_rows ? max_rows : n_rows;
    NEED(n >= 1 && n <= 65536 && n * 256 < (1ll << 32));
    NEED(all <= (1 << 22) || n == 1);
    // as many as the rows' blocks where those are few
    const int64_t need = rows == 1 ? 1 : (rows + 31) / 32 + 1;
    if (need <= 65536 && need * heads * seqs <= (1 << 22)) NEED(n == need);
  }
  std::printf("ok\n");
}
"""


def test_workgroups_are_bounded_whatever_the_hints(tmp_path):
    src, exe = tmp_path / "grid.cpp", tmp_path / "grid"
    src.write_text(HOST)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", ROOT, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout
