"""Without a GPU: the cache's indexes and bounds compiled for the host, every documented
refusal of the calls between the products, and the oracle they are measured with."""

import ctypes
import os
import subprocess

import numpy as np
import pytest

from oracle import decode as odec
from paper_2607_02893_amd import vbq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20  # an address that no refused call looks at


# ------------------------------------------------------------------ indexes

HOST = r"""
#include "paper_2607_02893_amd/csrc/vbq_cache.hpp"
#include <cstdio>
#include <cstdlib>
#include <vector>
using namespace vbq;
#define NEED(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); std::exit(1); } } while (0)
template <int D> void page() {
  // every code and scale of a page has a place of its own, and the places fill the page
  std::vector<int> bits(PageOf<D>::kBytes * 2, 0);
  for (int p = 0; p < kPage; ++p) {
    for (int d = 0; d < D; ++d) {
      const int k = key_word<D>(p, d / 32, (d / 8) % 4), v = value_word<D>(p / 32, d, slot_of(p) / 8);
      NEED(k % 4 == 0 && k >= 0 && k + 4 <= PageOf<D>::kValues);
      NEED(v % 4 == 0 && v >= PageOf<D>::kValues && v + 4 <= PageOf<D>::kKeyScales);
      ++bits[2 * k + code_bit(d % 8) / 4];
      ++bits[2 * v + code_bit(slot_of(p) % 8) / 4];
    }
    NEED(slot_of(p) >= 0 && slot_of(p) < 32);
    for (int g = 0; g < PageOf<D>::kGroups; ++g)
      for (int s : {PageOf<D>::kKeyScales, PageOf<D>::kValueScales})
        for (int n = 0; n < 4; ++n) ++bits[2 * (s + 128 * g + 2 * ((p & 32) + slot_of(p))) + n];
  }
  for (int n : bits) NEED(n == 1);
}
int main() {
  page<64>(); page<128>(); page<256>();
  // whatever the device arrays hold, rows stay in [0, n_rows) and positions in the table
  const int32_t odd[] = {-2147483647 - 1, -7, -1, 0, 1, 2, 5, 63, 64, 65, 2147483647};
  for (int32_t r0 : odd) for (int32_t r1 : odd) for (int32_t len : odd) for (int stride : {1, 2, 1 << 24}) for (int64_t rows : {1, 6, 70}) {
    const int32_t start[2] = {r0, r1}, lens[1] = {len};
    const Batch a{nullptr, start, lens, 1, stride, rows, 1};
    const Seq s = seq_of(a, 0);
    NEED(s.n >= 0 && s.row0 >= 0 && (s.n == 0 || s.row0 + s.n <= rows));
    NEED(s.end >= 0 && s.end <= (int64_t)stride * kPage && s.end <= 2147483647);
    if (len >= 0) NEED(s.pos0 == len - s.n);
  }
  for (int32_t id : odd) {
    const int32_t table[1] = {id};
    const Batch a{table, nullptr, nullptr, 1, 1, 1, 1};
    const int64_t got = page_id(a, 3, 0, 0);
    NEED(got == (id >= 0 && id < 3 ? id : -1));
  }
  std::printf("ok\n");
}
"""


def test_indexes_and_bounds_on_the_host(tmp_path):
    src, exe = tmp_path / "bounds.cpp", tmp_path / "bounds"
    src.write_text(HOST)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", ROOT, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout


# ------------------------------------------------------------------ refusals


def _desc(n_pages=4, heads=2, D=128):
    d = vbq.VbqKvDesc()
    return vbq.lib().vbq_kv_layout(n_pages, heads, D, ctypes.byref(d)), d


def test_layout():
    for D in (64, 128, 256):
        st, d = _desc(7, 3, D)
        assert st == 0 and d.page_bytes == 3 * 68 * D and d.total_bytes == 7 * 3 * 68 * D
    assert vbq.lib().vbq_kv_layout(1, 1, 64, None) == 1
    for args, want in (((0, 1, 64), 2), ((-1, 1, 64), 2), ((1 << 31, 1, 64), 2), ((1, 0, 64), 2), ((1, 1025, 64), 2),
                       ((1, 1, 0), 2), ((1, 1, 96), 10), ((1, 1, 512), 10), ((1, 1, 80), 10)):
        assert _desc(*args)[0] == want, args


def _batch(**kw):
    f = dict(n_seqs=2, table_stride=3, page_table=A, row_start=None, seq_len=A, n_rows=2, max_rows=1, max_len=100)
    f.update(kw)
    return vbq.VbqKvBatch(*[f[n] for n in ("n_seqs", "table_stride", "page_table", "row_start", "seq_len", "n_rows",
                                           "max_rows", "max_len")])


BAD_BATCHES = [(dict(n_seqs=-1), 2), (dict(n_seqs=65536, n_rows=65536), 2), (dict(n_rows=-1), 2), (dict(n_rows=3), 2), (dict(max_rows=0), 2),
               (dict(max_len=-1), 2), (dict(table_stride=0), 2), (dict(table_stride=(1 << 24) + 1), 2),
               (dict(row_start=A, n_rows=(1 << 30) + 1), 2), (dict(page_table=None), 1), (dict(seq_len=None), 1),
               (dict(page_table=A + 2), 7), (dict(seq_len=A + 1), 7), (dict(row_start=A + 2), 7)]


def _append(d, b, cache=A, type=0, k=A, ldk=256, hsk=128, v=A, ldv=256, hsv=128):
    return vbq.lib().vbq_kv_append(d, cache, b, type, k, ldk, hsk, v, ldv, hsv, None)


def _attention(d, b, cache=A, heads=4, scale=0.1, qt=1, q=A, ldq=512, hsq=128, ot=1, out=A, ldo=512, hso=128, ws=A, n=1 << 40):
    return vbq.lib().vbq_kv_attention(d, cache, b, heads, scale, qt, q, ldq, hsq, ot, out, ldo, hso, ws, n, None)


@pytest.mark.parametrize("fields,want", BAD_BATCHES)
def test_batches_are_refused_by_every_call(fields, want):
    d, b = ctypes.byref(_desc()[1]), ctypes.byref(_batch(**fields))
    n = ctypes.c_size_t(0)
    assert _append(d, b) == want
    assert _attention(d, b) == want
    assert vbq.lib().vbq_kv_dequant(d, A, b, A, A, None) == want
    assert vbq.lib().vbq_kv_attention_workspace_size(d, b, 4, ctypes.byref(n)) == want


def test_descriptors_are_refused_by_every_call():
    b = ctypes.byref(_batch())
    n = ctypes.c_size_t(0)
    for field, value in (("magic", 1), ("version", 2), ("n_pages", 0), ("n_heads", 0), ("head_dim", 100), ("page_bytes", 1),
                         ("total_bytes", 5)):
        _, desc = _desc()
        setattr(desc, field, value)
        d = ctypes.byref(desc)
        assert _append(d, b) == 8 and _attention(d, b) == 8 and vbq.lib().vbq_kv_dequant(d, A, b, A, A, None) == 8
        assert vbq.lib().vbq_kv_attention_workspace_size(d, b, 4, ctypes.byref(n)) == 8
    d = ctypes.byref(_desc()[1])
    assert _append(None, b) == 1 and _attention(None, b) == 1 and _append(d, None) == 1 and _attention(d, None) == 1
    assert vbq.lib().vbq_kv_dequant(None, A, b, A, A, None) == 1 and vbq.lib().vbq_kv_dequant(d, A, None, A, A, None) == 1
    assert vbq.lib().vbq_kv_attention_workspace_size(d, b, 4, None) == 1


def test_cache_call_arguments():
    d, b = ctypes.byref(_desc()[1]), ctypes.byref(_batch())
    for kw, want in ((dict(type=3), 10), (dict(cache=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(ldk=252), 2),
                     (dict(hsv=4), 2), (dict(ldv=-8), 2), (dict(hsk=1 << 41), 2), (dict(cache=A + 128), 7), (dict(k=A + 8), 7),
                     (dict(v=A + 4), 7)):
        assert _append(d, b, **kw) == want, kw
    for kw, want in ((dict(heads=3), 2), (dict(heads=0), 2), (dict(heads=2 * 257), 2), (dict(qt=3), 10), (dict(ot=-1), 10),
                     (dict(scale=float("nan")), 5), (dict(scale=float("inf")), 5), (dict(scale=0.0), 10), (dict(scale=-1.0), 10),
                     (dict(scale=1e30), 10), (dict(scale=2.0 ** 31), 10), (dict(scale=2.0 ** -61), 10), (dict(cache=None), 1), (dict(q=None), 1), (dict(out=None), 1), (dict(ldq=4), 2),
                     (dict(ldo=64), 2), (dict(hso=0), 2), (dict(q=A + 8), 7), (dict(out=A + 8), 7), (dict(cache=A + 16), 7)):
        assert _attention(d, b, **kw) == want, kw
    for args, want in (((None, A, A), 1), ((A, None, A), 1), ((A, A, None), 1), ((A + 8, A, A), 7), ((A, A + 4, A), 7), ((A, A, A + 8), 7)):
        assert vbq.lib().vbq_kv_dequant(d, args[0], b, args[1], args[2], None) == want
    many = ctypes.byref(_batch(row_start=A, n_rows=1 << 29))  # rows times query heads a kv head beyond 2^30
    assert _attention(d, many, heads=8) == 2
    # a long cache splits the positions: the workspace is asked for and checked
    long = ctypes.byref(_batch(table_stride=4096, max_len=4096 * 64))
    n = ctypes.c_size_t(0)
    assert vbq.lib().vbq_kv_attention_workspace_size(d, long, 4, ctypes.byref(n)) == 0 and n.value > 0
    assert _attention(d, long, ws=None) == 1 and _attention(d, long, ws=A + 8) == 7 and _attention(d, long, n=n.value - 1) == 7
    # nothing to do: nothing is looked at
    none = ctypes.byref(_batch(n_seqs=0, n_rows=0, page_table=None, seq_len=None))
    assert _append(d, none, k=None) == 0 and _attention(d, none, q=None) == 0
    assert vbq.lib().vbq_kv_dequant(d, None, none, None, None, None) == 0


def _norm(n=2, K=64, rt=0, r=A, ldr=64, yt=0, y=A, ldy=64, wt=0, w=A, eps=1e-5, h=A, ldh=64, xt=1, x=A, ldx=64):
    return vbq.lib().vbq_add_norm(n, K, rt, r, ldr, yt, y, ldy, wt, w, eps, h, ldh, xt, x, ldx, None)


def test_norm_arguments():
    for kw, want in ((dict(n=-1), 2), (dict(n=1 << 31), 2), (dict(K=0), 2), (dict(K=(1 << 24) + 1), 2), (dict(rt=3), 10), (dict(yt=5), 10),
                     (dict(wt=-1), 10), (dict(xt=9), 10), (dict(eps=float("nan")), 5), (dict(eps=float("inf")), 5), (dict(eps=-1.0), 10),
                     (dict(r=None), 1), (dict(x=None), 1), (dict(ldr=63), 2), (dict(ldx=63), 2), (dict(ldy=63), 2), (dict(ldh=0), 2),
                     (dict(ldx=1 << 41), 2), (dict(r=A + 2), 7), (dict(y=A + 1), 7), (dict(w=A + 2), 7), (dict(h=A + 2), 7), (dict(x=A + 1), 7)):
        assert _norm(**kw) == want, kw
    assert _norm(n=0, r=None, x=None) == 0


def _sample(M=2, V=100, t=0, z=A, ld=100, T=A, k=A, p=A, mp=A, u=A, tok=A, prob=A, ws=A, n=1 << 40):
    return vbq.lib().vbq_sample(M, V, t, z, ld, T, k, p, mp, u, tok, prob, ws, n, None)


def test_sample_arguments():
    for kw, want in ((dict(M=-1), 2), (dict(M=(1 << 20) + 1), 2), (dict(V=0), 2), (dict(V=(1 << 20) + 1, ld=1 << 21), 2), (dict(ld=99), 2),
                     (dict(ld=1 << 41), 2), (dict(t=3), 10), (dict(z=None), 1), (dict(u=None), 1), (dict(tok=None), 1),
                     (dict(z=A + 2), 7), (dict(t=1, z=A + 1), 7), (dict(T=A + 2), 7), (dict(k=A + 1), 7), (dict(p=A + 2), 7),
                     (dict(mp=A + 2), 7), (dict(u=A + 2), 7), (dict(tok=A + 2), 7), (dict(prob=A + 1), 7)):
        assert _sample(**kw) == want, kw
    assert _sample(M=0, z=None) == 0
    n = ctypes.c_size_t(0)
    f = vbq.lib().vbq_sample_workspace_size
    assert f(16, 128256, ctypes.byref(n)) == 0 and f(16, 128256, None) == 1 and f(-1, 5, ctypes.byref(n)) == 2 and f(1, 0, ctypes.byref(n)) == 2
    if n.value:
        assert _sample(M=16, V=128256, ld=128256, ws=None) == 1
        assert _sample(M=16, V=128256, ld=128256, ws=A + 8) == 7
        assert _sample(M=16, V=128256, ld=128256, n=n.value - 1) == 7


def test_binding_rejects_host_tensors():
    torch = pytest.importorskip("torch")
    z = torch.zeros((2, 64))
    with pytest.raises(ValueError, match="GPU tensor"):
        vbq.add_norm(z)
    with pytest.raises(ValueError, match="GPU tensor"):
        vbq.sample(z, torch.zeros(2))
    with pytest.raises(ValueError, match="GPU tensor"):
        vbq.KVBatch(torch.zeros((1, 1), dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError, match="overlap"):
        vbq._spread(torch.zeros(64).expand(4, 64), "x")
    with pytest.raises(ValueError, match="overlap"):
        vbq._spread(torch.zeros(64).as_strided((3, 4), (2, 1)), "x")
    vbq._spread(torch.zeros((4, 2, 8)).transpose(0, 1), "x")


# ------------------------------------------------------------------ the oracle


def test_oracle_quantizer_and_rounding():
    rng = np.random.default_rng(1)
    w = rng.standard_normal((3, 128)) * np.array([[1.0], [1e-3], [50.0]])
    w[0, :64] = 0.0
    q, s = odec.kv_quantize(w)
    assert s[0, 0] == 0 and not q[0, :64].any() and np.abs(q).max() == 7
    assert np.all(np.abs(odec.kv_values(w) - w) <= np.repeat(s, 64, axis=1) * 0.51 + 1e-12)
    assert odec.round_to(1.0 + 2.0 ** -9, "bf16") == 1.0 and odec.round_to(1.0 + 3 * 2.0 ** -8, "bf16") == 1.0 + 2.0 ** -6
    assert odec.round_to(1.0 + 2.0 ** -11, "f16") == 1.0


def test_oracle_attention_closed_forms():
    keys, values = np.zeros((3, 1, 64)), np.arange(3.0)[:, None, None] * np.ones((3, 1, 64))
    out, _ = odec.attention(np.ones((4, 2, 64)), keys, values, 1.0, 3)  # rows at positions -1, 0, 1, 2
    assert np.allclose(out[:, 0, 0], [0.0, 0.0, 0.5, 1.0])


def test_oracle_sample_closed_forms():
    z = np.log(np.array([1.0, 4.0, 2.0, 4.0, 1.0]))
    for u, tok in ((0.0, 0), (0.09, 1), (0.2, 1), (0.5, 2), (0.8, 3), (0.95, 4)):
        assert odec.sample(z, u)[0] == tok
    assert odec.sample(z, 0.99, top_k=1)[:2] == (1, 1.0)          # the lower index of equals
    assert odec.sample(z, 0.99, top_k=2)[0] == 3
    assert odec.sample(z, 0.99, top_p=0.5)[0] == 3                # 4 + 4 of 12 is needed to reach half
    assert odec.sample(z, 0.99, top_p=0.3)[0] == 1
    assert odec.sample(z, 0.99, min_p=0.5)[0] == 3 and odec.sample(z, 0.7, min_p=0.6)[0] == 3
    assert odec.sample(z, 0.3, temperature=0.0)[:2] == (1, 1.0)
    assert odec.sample([np.nan, -np.inf], 0.3)[:2] == (-1, 0.0)
    assert odec.sample([np.nan, np.inf, 3.0, np.inf], 0.6)[:2] == (3, 0.5)
