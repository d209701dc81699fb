"""A value group that is NaN gives NaN to every row that sees its position, however little
the position weighs and however the positions are split over waves and parts."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_cache import Case, _say  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vbq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2607_02893_amd import vbq as v
    return v


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("L,rows", [(50, 1), (100, 1), (300, 3), (3000, 1), (5000, 40)])
def test_a_nan_value_of_negligible_weight(vbq, d, L, rows):
    rng = np.random.default_rng(L + d)
    c = Case(vbq, rng, [L], 1, d, kv="f32")
    q = torch.zeros((rows, 2, d), dtype=torch.float16, device="cuda")
    q[:, :, d - 3] = 20.0
    for at, big in ((0, L - rows), (L - rows, 0), (L // 2, 0), (0, L // 2)):
        if at == big:
            continue
        k, v = torch.zeros_like(c.k[0]), c.v[0].clone()
        k[big, 0, d - 3] = 20.0               # its score is 400, the others' 0
        v[at, 0, 7] = float("nan")
        c.cache.append(k, v, vbq.KVBatch(c.t, c.l, max_rows=L))
        for max_len in (None, 1, L, 100 * L):
            _say(f"nan d={d} L={L} rows={rows} at={at} big={big} max_len={max_len}")
            out = c.cache.attention(q, c.batch([rows], max_len=max_len), scale=1.0, out_dtype=torch.float32)
            assert torch.isnan(out[:, :, :64]).all() and torch.isfinite(out[:, :, 64:]).all()
