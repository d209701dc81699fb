"""Hints so far off that the parts' sums would outgrow the workspace: the same result in fewer parts."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_cache import Case, _check_attention, _rows, _say  # noqa: E402

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
