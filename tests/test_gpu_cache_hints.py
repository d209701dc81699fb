"""Hints so far off that the parts' sums would outgrow the workspace, or the grid all bounds: the same
result in fewer parts, the same bytes from fewer workgroups."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import decode as odec  # noqa: E402
from tests.test_gpu_cache import Case, _check_attention, _dev, _np, _rows, _say  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vbq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2607_02893_amd import vbq as v
    return v


@pytest.mark.parametrize("d,group,lens,rows,max_len", [
    (64, 64, [70], [70], 2 ** 31 - 1),          # one part is left of 64, all else empty
    (64, 32, [1300], [500], 16400),             # 16 of 17, two in use
    (128, 32, [600, 64], [300, 1], 100000),
])
def test_many_rows_said_to_be_one(vbq, d, group, lens, rows, max_len):
    rng = np.random.default_rng(d + group)
    _say(f"hints d={d} group={group} lens={lens} rows={rows} max_len={max_len}")
    c = Case(vbq, rng, lens, 1, d)
    q = _rows(rng, sum(rows), group, d, "f16")
    b = c.batch(rows, max_rows=1, max_len=max_len)
    need = c.cache.attention_workspace_size(b, group)
    assert 0 < need <= (1 << 18) * (d + 2) * 4
    out = c.cache.attention(q, b, out_dtype=torch.float32)
    _check_attention(out, q, c, rows, d ** -0.5, "f32", what="hints")


def test_many_sequences_and_a_far_hint(vbq):
    """Each workgroup goes on to the blocks that a smaller grid leaves: two long sequences of 4000, one row elsewhere."""
    rng = np.random.default_rng(40)
    n, hkv, d = 4000, 64, 64
    rows = np.zeros(n, dtype=np.int64)
    rows[[7, 3999]] = [900, 700]
    rows[100] = 1
    starts = np.concatenate([[0], np.cumsum(rows)])
    total = int(starts[-1])
    table = np.full((n, 15), -1, dtype=np.int32)
    table[7], table[3999, :11], table[100, 0] = np.arange(15), np.arange(15, 26), 26
    lens = rows.astype(np.int32)
    few = vbq.KVCache(27, hkv, d)
    k, v = _rows(rng, total, hkv, d, "f16"), _rows(rng, total, hkv, d, "f16")
    far = vbq.KVBatch(_dev(table), _dev(lens), _dev(starts), n_rows=total, max_rows=2 ** 31 - 1)
    _say("append, 4000 sequences, far hint")
    few.append(k, v, far)
    dk, dv = few.dequant(far)
    assert np.array_equal(_np(dk), odec.kv_values(_np(k))) and np.array_equal(_np(dv), odec.kv_values(_np(v)))
