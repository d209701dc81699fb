"""What a row does not see does not reach it: the keys and values of later tokens, however
large, change no bit of an earlier row's result, and the row keeps the precision that its own
positions give it (the bound of test_gpu_cache, taken over the positions that it sees)."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import decode as odec  # noqa: E402
from tests.test_gpu_cache import TYPES, Case, _check_attention, _np, _rows, _say  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vbq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2607_02893_amd import vbq as v
    return v


class Prefix:
    """The first `n` positions of every sequence."""

    def __init__(self, keys, values, lens, hkv, d):
        self.keys, self.values = [k[:n] for k, n in zip(keys, lens)], [v[:n] for v, n in zip(values, lens)]
        self.lens, self.hkv, self.d = lens, hkv, d


SHAPES = [  # d, hkv, group, lens, rows
    (64, 1, 2, [21], [2]),
    (128, 2, 4, [21, 40], [2, 17]),
    (256, 1, 2, [21, 130], [5, 70]),
    (64, 8, 4, [100, 131], [64, 70]),     # 32 rows of a workgroup
    (128, 8, 4, [100, 131], [64, 70]),
    (128, 1, 2, [2500], [70]),            # split positions
    (256, 1, 1, [4150], [20]),
    (64, 8, 4, [4200, 300], [64, 60]),    # both
]


@pytest.mark.parametrize("qt", ["f16", "f32"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_later_tokens_change_nothing(vbq, shape, qt):
    d, hkv, group, lens, rows = SHAPES[shape]
    rng = np.random.default_rng(300 + shape)
    _say(f"hidden d={d} hkv={hkv} group={group} lens={lens} rows={rows} {qt}")
    c = Case(vbq, rng, lens, hkv, d, kv="f32")
    k, v = [x.clone() for x in c.k], [x * 1e-4 for x in c.v]
    values = [odec.kv_values(_np(x)) for x in v]
    q = _rows(rng, sum(rows), hkv * group, d, qt)
    starts = np.concatenate([[0], np.cumsum(rows)])
    b = c.batch(rows)

    def fill(k, v):
        for i, n in enumerate(lens):
            one = vbq.KVBatch(c.t[i:i + 1].contiguous(), c.l[i:i + 1].contiguous(), max_rows=n)
            c.cache.append(k[i], v[i], one)

    fill(k, v)
    plain = c.cache.attention(q, b, out_dtype=torch.float32)
    for share in (0.0, 0.5):
        hidden = [max(1, int(n * share)) for n in rows]  # so many of the last tokens are changed
        keep = [n - h for n, h in zip(rows, hidden)]
        for large in (6.0e4, 4.0e5, float("nan"), 0.0):
            k2, v2 = [x.clone() for x in k], [x.clone() for x in v]
            for i, h in enumerate(hidden):
                v2[i][-h:] = large * torch.sign(v2[i][-h:])
                k2[i][-h:] *= 3.0
            fill(k2, v2)
            out = c.cache.attention(q, b, out_dtype=torch.float32)
            at = np.concatenate([np.arange(starts[i], starts[i] + n) for i, n in enumerate(keep)])
            before = Prefix(c.keys, values, [n - h for n, h in zip(lens, hidden)], hkv, d)
            _check_attention(out[at], q[at], before, keep, d ** -0.5, "f32", what=f"last {hidden} are {large}")
            assert torch.equal(out[at], plain[at]), f"last {hidden} are {large}"


def test_a_row_alone_and_among_others(vbq):
    """The last row sees the large value, the rows before it do not: each as precise as its own positions allow."""
    rng = np.random.default_rng(320)
    L, n = 30, 10
    c = Case(vbq, rng, [L], 1, 128, kv="bf16")
    v = (c.v[0] * 1e-5).to(TYPES["bf16"])
    v[-1] = 4.0e5
    c.cache.append(c.k[0], v, vbq.KVBatch(c.t, c.l, max_rows=L))
    values = [odec.kv_values(_np(v))]
    q = _rows(rng, n, 4, 128, "f16")
    out = c.cache.attention(q, c.batch([n]), out_dtype=torch.float32)
    for r in range(n):
        seen = Prefix(c.keys, values, [L - n + r + 1], 1, 128)
        _check_attention(out[r:r + 1], q[r:r + 1], seen, [1], 128 ** -0.5, "f32", what=f"row {r}")
