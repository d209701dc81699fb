"""The 4-bit cache and the attention over it against the oracle.

Append and dequant are exact: the bytes of every appended position are the oracle's
levels and scales, and all other bytes of the cache stay as they were.

Attention, tolerance (u = 2^-24).  With the cache's exact values, the calls' errors are:
  * a score: sums of D products in fp32 on the matrix cores.  A group's sum has terms of
    at most 15 |q_i| and starts at 8 |sum q|, so 32 u of 23 sum |q_i| s covers any order
    of the 64 additions and the cores' alignment of 32 terms (a 2^-24 share of the largest
    each).  fp32 queries as two fp16 terms are off by 2^-22, included with another 8 u of
    7 sum |q_i| s; times the scale this is d.  The power of two's argument is rounded
    once, at most 2^-23 of (|score| + its largest) log2 e;
  * so a weight is off by at most e = 2 d + 2^-22 (|score| + max |score|) + 2^-21 relative
    (v_exp_f32 is within 2^-22), and its product with the value scale by half a step of fp16 more,
    2^-11, or, below fp16's normals, by 2^-25 of a unit where the largest weight times the
    largest scale is at least 2^6: 2^-31 of the largest value scale a position, at most 7
    levels of it;
  * the sum of weights by e and the fp32 sum, the weighted sums by the cores' fp32 (L + 32 terms
    aligned: 2^-20 allowed, L below 2^15 here), so
    |out - o| <= (2^-11 + 2 e + 2^-19) A + 2^-28 L smax + eps/2 |o|,
    A the weighted mean of |v|, eps/2 the output type's half step.
With q = 0 all weights are 1 and 1 times a scale is exact: there the first term is 2^-19 A, which
tells one missing or doubled position among thousands.
"""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import decode as odec  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def vbq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2607_02893_amd import vbq as v
    return v


def _say(msg):
    print(msg, flush=True)


def _rows(rng, n, h, d, dtype):
    w = rng.standard_normal((n, h, d)) * np.exp(0.5 * rng.standard_normal((h, d)))
    return torch.from_numpy(w).to(TYPES[dtype]).cuda()


def _np(t):
    return t.double().cpu().numpy()


def _table(rng, lens, spare=1, stride=None):
    need = [(max(l, 0) + 63) // 64 for l in lens]
    order = rng.permutation(sum(need) + spare)
    table = np.full((len(lens), stride or max(1, max(need))), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return sum(need) + spare, table


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


class Case:
    """A cache filled through append, its memory poisoned first, and what it should hold."""

    def __init__(self, vbq, rng, lens, hkv, d, kv="f16", poison=0xFF, stride=None):
        self.vbq, self.lens, self.hkv, self.d = vbq, lens, hkv, d
        n_pages, self.table = _table(rng, lens, stride=stride)
        self.cache = vbq.KVCache(n_pages, hkv, d)
        self.cache.data.fill_(poison)
        self.k = [_rows(rng, l, hkv, d, kv) for l in lens]
        self.v = [_rows(rng, l, hkv, d, kv) for l in lens]
        self.t, self.l = _dev(self.table), _dev(lens)
        starts = np.concatenate([[0], np.cumsum(lens)])
        if starts[-1]:
            b = vbq.KVBatch(self.t, self.l, _dev(starts), n_rows=int(starts[-1]), max_rows=max(max(lens), 1))
            self.cache.append(torch.cat(self.k), torch.cat(self.v), b)
        self.keys = [odec.kv_values(_np(k)) if k.shape[0] else _np(k) for k in self.k]
        self.values = [odec.kv_values(_np(v)) if v.shape[0] else _np(v) for v in self.v]

    def batch(self, rows, **kw):
        starts = np.concatenate([[0], np.cumsum(rows)])
        kw.setdefault("max_rows", max(1, max(rows)))
        return self.vbq.KVBatch(self.t, self.l, _dev(starts), n_rows=int(starts[-1]), **kw)


def _check_attention(got, q, case, rows, scale, out_type, seqs=None, what=""):
    """Every row against the oracle with the bound derived above; returns the worst share of it."""
    at, worst = 0, 0.0
    for b, n in enumerate(rows):
        keys, values, L = case.keys[b], case.values[b], case.lens[b]
        x = _np(q[at:at + n])
        ref, size = odec.attention(x, keys, values, scale, L)
        group = x.shape[1] // case.hkv
        if L:
            ks = np.abs(keys).max(axis=0) / 7.0  # per channel, at least the scale's levels reach it
            s_groups = np.repeat(np.abs(keys).reshape(L, case.hkv, -1, 64).max(axis=(0, 3)) / 7.0, 64, axis=-1)
            del ks
            weight = np.repeat(np.abs(np.ones((1, case.hkv, case.d)) * s_groups[None]), group, axis=1)
            reach = (np.abs(x) * weight).sum(axis=-1, keepdims=True)
            d = scale * 2.0 ** -24 * (32 * 23 + 8 * 7) * reach
            top = scale * 7 * reach
            e = 2 * d + 2.0 ** -22 * 2 * top + 2.0 ** -21
            smax = np.abs(values).max() / 7.0
        else:
            e, smax = np.zeros((n, x.shape[1], 1)), 0.0
        flat = 0.0 if not x.any() else 2.0 ** -11
        bound = (flat + 2 * e + 2.0 ** -19) * size + 2.0 ** -28 * L * smax + HALF_STEP[out_type] * np.abs(ref)
        bound = bound + (2.0 ** -25 if out_type == "f16" else 0.0) + 1e-30
        err = np.abs(_np(got[at:at + n]) - ref)
        assert np.isfinite(_np(got[at:at + n])).all(), f"{what} sequence {b}: not finite"
        bad = err > bound
        assert not bad.any(), f"{what} sequence {b} (L={L}): {bad.sum()} of {bad.size} off, first {np.argwhere(bad)[0]}, worst {(err / bound).max()}"
        worst = max(worst, float((err / bound).max()) if err.size else 0.0)
        at += n
    return worst


# ------------------------------------------------------------------ append, dequant


@pytest.mark.parametrize("kv", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,hkv", [(64, 3), (128, 2), (256, 1)])
def test_append_writes_the_oracles_bytes_and_no_others(vbq, d, hkv, kv):
    rng = np.random.default_rng(d + hkv)
    lens, rows = [70, 1, 33, 0, 128, 31], [70, 1, 5, 0, 65, 30]
    _say(f"append d={d} hkv={hkv} {kv}")
    n_pages, table = _table(rng, lens)
    cache = vbq.KVCache(n_pages, hkv, d)
    before = rng.integers(0, 256, cache.nbytes, dtype=np.uint8)
    cache.data.copy_(torch.from_numpy(before))
    starts = np.concatenate([[0], np.cumsum(rows)])
    k, v = _rows(rng, sum(rows), hkv, d, kv), _rows(rng, sum(rows), hkv, d, kv)
    k[3, 0, :64] = 0.0                                   # an all-zero group
    k[4, 0, :64] = torch.tensor([7.0, -3.5, 0.5, -0.5, 2.5, 1.5, -7.0, 0.25] * 8)  # ties
    v[5, hkv - 1, :64] *= 1e-7                           # a subnormal or zero scale
    b = vbq.KVBatch(_dev(table), _dev(lens), _dev(starts), n_rows=sum(rows), max_rows=max(rows))
    cache.append(k, v, b)
    got = cache.data.cpu().numpy().reshape(n_pages, -1)
    kq, ks = odec.kv_quantize(_np(k))
    vq, vs = odec.kv_quantize(_np(v))
    written = [set() for _ in range(n_pages)]
    for s, (l, n) in enumerate(zip(lens, rows)):
        for r in range(n):
            p, row = l - n + r, starts[s] + r
            page = table[s, p // 64]
            written[page].add(p % 64)
            for h in range(hkv):
                a = odec.page_position(got[page], h, d, p % 64)
                for x, y in zip(a, (kq[row, h], ks[row, h], vq[row, h], vs[row, h])):
                    assert np.array_equal(x, y), f"sequence {s} position {p} head {h}"
    old = before.reshape(n_pages, -1)
    for page in range(n_pages):
        for p in set(range(64)) - written[page]:
            for h in range(hkv):
                for x, y in zip(odec.page_position(got[page], h, d, p), odec.page_position(old[page], h, d, p)):
                    assert np.array_equal(x, y, equal_nan=True), f"page {page} position {p} changed"
    dk, dv = cache.dequant(b)
    assert np.array_equal(_np(dk), odec.kv_values(_np(k))) and np.array_equal(_np(dv), odec.kv_values(_np(v)))


def test_append_one_token_at_a_time_is_append_at_once(vbq):
    rng = np.random.default_rng(3)
    lens, d, hkv = [67, 130], 128, 2
    c = Case(vbq, rng, lens, hkv, d, poison=0x5A)
    one = vbq.KVCache(c.cache.n_pages, hkv, d)
    one.data.fill_(0x5A)
    for p in range(max(lens)):
        live = [b for b in range(2) if p < lens[b]]
        k = torch.stack([c.k[b][p] for b in live])
        v = torch.stack([c.v[b][p] for b in live])
        one.append(k, v, vbq.KVBatch(c.t[live].contiguous(), _dev([p + 1] * len(live))))
    assert torch.equal(one.data, c.cache.data)


def test_append_takes_views_of_a_fused_projection(vbq):
    rng = np.random.default_rng(4)
    d, hkv, hq, n = 64, 2, 4, 3
    y = torch.from_numpy(rng.standard_normal((n, (hq + 2 * hkv) * d + 8))).float().cuda()
    heads = y[:, :(hq + 2 * hkv) * d].unflatten(1, (hq + 2 * hkv, d))
    k, v = heads[:, hq:hq + hkv], heads[:, hq + hkv:]
    a, b = vbq.KVCache(n, hkv, d), vbq.KVCache(n, hkv, d)
    batch = vbq.KVBatch(_dev([[0], [1], [2]]), _dev([1, 5, 64]))
    a.append(k, v, batch)
    b.append(k.contiguous(), v.contiguous(), batch)
    assert torch.equal(a.data, b.data) and bool(a.data.any())
    # heads outermost: strides in the other order
    a.data.zero_()
    a.append(k.transpose(0, 1).contiguous().transpose(0, 1), v, batch)
    assert torch.equal(a.data, b.data)


def test_rows_without_a_place_are_dropped(vbq):
    rng = np.random.default_rng(5)
    d, hkv = 128, 1
    cache = vbq.KVCache(3, hkv, d)
    cache.data.fill_(0x33)
    k, v = _rows(rng, 9, hkv, d, "f16"), _rows(rng, 9, hkv, d, "f16")
    # sequence 0: three rows, length 1 (two before position 0); 1: no page; 2: page beyond the
    # cache; 3: longer than its table
    table, lens = [[0], [-1], [3], [2]], [1, 4, 4, 65]
    batch = vbq.KVBatch(_dev(table), _dev(lens), _dev([1, 4, 5, 6, 8]), n_rows=9, max_rows=3)
    cache.append(k, v, batch)
    data = cache.data.cpu().numpy().reshape(3, -1)
    assert (data[1] == 0x33).all()
    dk = torch.full((9, hkv, d), 77.0, device="cuda")
    dv = dk.clone()
    cache.dequant(batch, dk, dv)
    want = np.full((9, hkv, d), 77.0)
    want[3] = odec.kv_values(_np(k))[3]   # sequence 0, position 0
    want[6] = odec.kv_values(_np(k))[6]   # sequence 3, position 63; its next row is past the table
    assert np.array_equal(_np(dk), want)
    out = torch.full((9, 2, d), 5.0, device="cuda", dtype=torch.float16)
    cache.attention(_rows(rng, 9, 2, d, "f16"), batch, out=out)
    got = _np(out)
    assert (got[[0, 8]] == 5.0).all(), "rows of no sequence"
    assert (got[[1, 2, 4, 5]] == 0.0).all(), "rows that see nothing"
    assert np.array_equal(got[3], np.repeat(odec.round_to(odec.kv_values(_np(v))[3], "f16"), 2, axis=0)) or \
        np.abs(got[3] - odec.kv_values(_np(v))[3]).max() < 2.0 ** -9 * np.abs(got[3]).max()


def test_not_finite_rows_stay_with_their_heads(vbq):
    rng = np.random.default_rng(6)
    d, lens = 128, [40]
    for bad in (float("nan"), float("inf"), -float("inf"), 1e30):
        c = Case(vbq, rng, lens, 2, d, kv="f32")
        k, v = c.k[0][39:].clone(), c.v[0][39:].clone()
        v[0, 1, 5] = bad
        c.cache.append(k, v, vbq.KVBatch(c.t, c.l))
        q = _rows(rng, 2, 2, d, "f16")
        out = _np(c.cache.attention(q, c.batch([2]), out_dtype=torch.float32))
        assert np.isfinite(out[:, 0]).all() and np.isfinite(out[0]).all(), "a position the row does not see"
        assert not np.isfinite(out[1, 1, :64]).any() and np.isfinite(out[1, 1, 64:]).all()
        k[0, 1, 70] = bad
        v = c.v[0][39:].clone()
        c.cache.append(k, v, vbq.KVBatch(c.t, c.l))
        out = _np(c.cache.attention(q, c.batch([2]), out_dtype=torch.float32))
        assert np.isfinite(out[:, 0]).all() and np.isfinite(out[0]).all() and np.isnan(out[1, 1]).all()


# ------------------------------------------------------------------ attention

SHAPES = [  # d, hkv, group, lens, rows
    (64, 2, 1, [1, 31, 32, 33, 63, 64, 65, 0, 127], [1] * 9),
    (128, 2, 4, [1, 16, 17, 48, 96, 129, 200], [1] * 7),
    (256, 1, 3, [5, 64, 100, 257], [1, 1, 1, 1]),
    (128, 1, 8, [9, 70, 66, 300, 3], [2, 3, 5, 7, 5]),        # more rows than 16, and rows before position 0
    (64, 1, 16, [80, 130, 64], [4, 2, 1]),
    (128, 1, 20, [90, 33], [1, 3]),                           # a group that is no divisor of 16
    (256, 2, 2, [40, 129], [9, 1]),
    (128, 2, 4, [150, 64, 97, 20], [150, 17, 1, 40]),
    (64, 1, 1, [200, 333], [200, 90]),
    (256, 1, 4, [130, 70], [60, 33]),
    (128, 4, 1, [3000, 17, 0, 1111], [1, 1, 0, 1]),           # split positions
    (64, 1, 6, [5001], [3]),
    (256, 1, 2, [2050], [1]),
    (128, 1, 2, [2500], [70]),
    (64, 8, 4, [100, 90], [64, 50]),                          # many tiles: 32 rows of a workgroup
    (128, 8, 4, [70, 131], [70, 40]),
    (64, 8, 4, [4200, 300], [64, 60]),                        # the same, split
    (128, 16, 2, [1500, 40, 0, 200], [33, 40, 3, 64]),
    (64, 1, 256, [70], [1]),                                  # the largest group
]


@pytest.mark.parametrize("qt,ot", [("f16", "f32"), ("f32", "f16"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention_matches_the_oracle(vbq, shape, qt, ot):
    d, hkv, group, lens, rows = SHAPES[shape]
    rng = np.random.default_rng(100 + shape)
    _say(f"attention d={d} hkv={hkv} group={group} lens={lens} rows={rows} {qt}->{ot}")
    c = Case(vbq, rng, lens, hkv, d)
    q = _rows(rng, sum(rows), hkv * group, d, qt)
    out = c.cache.attention(q, c.batch(rows), out_dtype=TYPES[ot])
    worst = _check_attention(out, q, c, rows, 1.0 / math.sqrt(d), ot, what=f"shape {shape} {qt}->{ot}")
    _say(f"  worst {worst:.3f} of the bound")
    # the same bits again
    assert torch.equal(out, c.cache.attention(q, c.batch(rows), out_dtype=TYPES[ot]))


@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_equal_weights_are_the_mean(vbq, shape):
    """q = 0: every position counts once, and the result is exact but for fp32 sums."""
    d, hkv, group, lens, rows = SHAPES[shape]
    rng = np.random.default_rng(200 + shape)
    _say(f"mean d={d} lens={lens} rows={rows}")
    c = Case(vbq, rng, lens, hkv, d)
    q = torch.zeros((sum(rows), hkv * group, d), dtype=torch.float16, device="cuda")
    out = c.cache.attention(q, c.batch(rows), out_dtype=torch.float32)
    _check_attention(out, q, c, rows, 0.125, "f32", what=f"shape {shape}")


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("rows", [1, 80])
def test_one_position_is_found(vbq, d, rows):
    """Keys with one large channel at one position: the row gets that position's value."""
    rng = np.random.default_rng(7 + d)
    L = 500
    lens = [L]
    for at in (0, 15, 16, 31, 32, 63, 64, 300, L - rows):
        c = Case(vbq, rng, lens, 1, d)
        k = c.k[0].clone()
        k[:] = 0.0
        k[at, 0, d - 3] = 100.0
        c.cache.append(k, c.v[0], vbq.KVBatch(c.t, c.l, max_rows=L))
        q = torch.zeros((rows, 2, d), dtype=torch.float16, device="cuda")
        q[:, :, d - 3] = 100.0
        out = _np(c.cache.attention(q, c.batch([rows]), scale=1.0, out_dtype=torch.float32))
        want = c.values[0][at, 0]
        # its weight is 1, the others e^-10000; the weight times the scale is exact up to its rounding
        assert np.abs(out - want).max() <= 2.0 ** -11 * np.abs(want).max() + 1e-12, (d, at)


def test_scores_that_grow_and_scales_that_vary(vbq):
    """Later keys beat earlier ones again and again, value scales span 2^-20 .. 2^8, scores reach thousands."""
    rng = np.random.default_rng(8)
    d, L = 128, 700
    for rows in (1, 40):
        c = Case(vbq, rng, [L], 1, d, kv="f32")
        k = c.k[0].clone()
        v = c.v[0].clone()
        k *= torch.linspace(0.01, 6.0, L, device="cuda")[:, None, None]
        v *= torch.exp2(torch.linspace(-17.0, 8.0, L, device="cuda"))[:, None, None]
        c.cache.append(k, v, vbq.KVBatch(c.t, c.l, max_rows=L))
        c.keys, c.values = [odec.kv_values(_np(k))], [odec.kv_values(_np(v))]
        for factor, scale in ((1.0, 0.05), (1e4, 1e-5), (1e-6, 1e4), (300.0, 0.02)):
            q = _rows(rng, rows, 3, d, "f32") * factor
            out = c.cache.attention(q, c.batch([rows]), scale=scale, out_dtype=torch.float32)
            _check_attention(out, q, c, [rows], scale, "f32", what=f"factor {factor}")
        # small scales at the positions that count, large ones where nothing looks
        v2 = v.flip(0).contiguous()
        c.cache.append(k, v2, vbq.KVBatch(c.t, c.l, max_rows=L))
        c.values = [odec.kv_values(_np(v2))]
        q = _rows(rng, rows, 3, d, "f32")
        out = c.cache.attention(q, c.batch([rows]), scale=0.02, out_dtype=torch.float32)
        _check_attention(out, q, c, [rows], 0.02, "f32", what="flipped")


def test_hints_do_not_change_the_result(vbq):
    """max_rows and max_len of a call with `rows` size the launch only."""
    rng = np.random.default_rng(9)
    lens, rows = [700, 65, 300], [90, 1, 33]
    c = Case(vbq, rng, lens, 2, 128)
    q = _rows(rng, sum(rows), 4, 128, "f16")
    for max_rows, max_len in ((1, 0), (1, 64), (7, 100000), (90, 1), (1000, 5), (3, 2 ** 31 - 1)):
        _say(f"hints {max_rows} {max_len}")
        b = c.batch(rows, max_rows=max_rows, max_len=max_len)
        out = c.cache.attention(q, b, out_dtype=torch.float32)
        _check_attention(out, q, c, rows, 128 ** -0.5, "f32", what=f"hints {max_rows} {max_len}")
        a = vbq.KVCache(c.cache.n_pages, 2, 128)
        a.append(_rows(np.random.default_rng(1), sum(rows), 2, 128, "f16"), _rows(np.random.default_rng(2), sum(rows), 2, 128, "f16"), b)
        dk, _ = a.dequant(b)
        assert np.array_equal(_np(dk), odec.kv_values(_np(_rows(np.random.default_rng(1), sum(rows), 2, 128, "f16"))))


def test_strides_of_queries_and_results(vbq):
    rng = np.random.default_rng(10)
    d, lens, rows = 64, [100, 50], [3, 2]
    c = Case(vbq, rng, lens, 2, d)
    wide = torch.from_numpy(rng.standard_normal((5, 4 * d + 24))).half().cuda()
    q = wide[:, 8:8 + 4 * d].unflatten(1, (4, d))
    out = torch.full((4, 5, d + 8), 9.0, dtype=torch.float32, device="cuda")
    view = out.permute(1, 0, 2)[:, :, :d]          # heads outermost, padded
    c.cache.attention(q, c.batch(rows), out=view)
    _check_attention(view, q, c, rows, d ** -0.5, "f32", what="strided")
    assert (out[:, :, d:] == 9.0).all()
    with pytest.raises(vbq.VbqError):
        c.cache.attention(wide[:, 4:4 + 4 * d].unflatten(1, (4, d)), c.batch(rows))  # 8 bytes off 16
    with pytest.raises(ValueError):
        c.cache.attention(q, c.batch(rows), out=torch.empty((1, 4, d), device="cuda").expand(5, 4, d))
    with pytest.raises(ValueError):
        c.cache.attention(q.transpose(1, 2), c.batch(rows))


def test_shared_pages(vbq):
    """Two sequences whose first pages are the same."""
    rng = np.random.default_rng(11)
    c = Case(vbq, rng, [128 + 20, 128 + 33], 1, 128)
    t = c.table.copy()
    t[1, :2] = t[0, :2]
    c.t = _dev(t)
    c.keys[1] = np.concatenate([c.keys[0][:128], c.keys[1][128:]])
    c.values[1] = np.concatenate([c.values[0][:128], c.values[1][128:]])
    q = _rows(rng, 3, 4, 128, "f16")
    out = c.cache.attention(q, c.batch([1, 2]), out_dtype=torch.float32)
    _check_attention(out, q, c, [1, 2], 128 ** -0.5, "f32", what="shared")


def test_pages_past_32_bit_offsets(vbq):
    """A cache beyond 4 GiB, its last pages in use."""
    rng = np.random.default_rng(12)
    d, hkv = 256, 8
    per = 68 * d * hkv
    n_pages = (1 << 32) // per + 40
    cache = vbq.KVCache(n_pages, hkv, d)
    L = 200
    table = _dev([[n_pages - 1, 0, n_pages - 30, n_pages - 2]])
    k, v = _rows(rng, L, hkv, d, "f16"), _rows(rng, L, hkv, d, "f16")
    b = vbq.KVBatch(table, _dev([L]), max_rows=L)
    cache.append(k, v, b)
    dk, dv = cache.dequant(b)
    keys, values = odec.kv_values(_np(k)), odec.kv_values(_np(v))
    assert np.array_equal(_np(dk), keys) and np.array_equal(_np(dv), values)

    class C:
        pass
    c = C()
    c.keys, c.values, c.lens, c.hkv, c.d = [keys], [values], [L], hkv, d
    q = _rows(rng, 1, hkv, d, "f16")
    out = cache.attention(q, vbq.KVBatch(table, _dev([L])), out_dtype=torch.float32)
    _check_attention(out, q, c, [1], d ** -0.5, "f32", what="far pages")


def test_streams_workspaces_and_graphs(vbq):
    rng = np.random.default_rng(13)
    c = Case(vbq, rng, [3000, 900], 2, 128)
    q = _rows(rng, 2, 8, 128, "f16")
    b = c.batch([1, 1])
    want = c.cache.attention(q, b)
    need = c.cache.attention_workspace_size(b, 8)
    assert need > 0, "this case is meant to split the positions"
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.cache.attention(q, b, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    with pytest.raises(vbq.VbqError):
        c.cache.attention(q, b, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    # two graphs on one workspace, lengths that change between replays
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    outs, graphs = [torch.empty_like(q), torch.empty_like(q)], []
    k, v = [_rows(rng, 2, 2, 128, "f16") for _ in range(2)], [_rows(rng, 2, 2, 128, "f16") for _ in range(2)]
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.cache.append(k[i], v[i], b)
            c.cache.attention(q, b, out=outs[i], workspace=ws)
        graphs.append(g)
    for step, lens in enumerate(([3000, 900], [2999, 64], [130, 1], [3000, 899])):
        c.l.copy_(_dev(lens))
        for i in range(2):
            outs[i].fill_(3.0)
            graphs[i].replay()
            torch.cuda.synchronize()
            c.cache.append(k[i], v[i], b)
            eager = c.cache.attention(q, b)
            assert torch.equal(outs[i], eager), (step, i)
            junk = torch.randn(1 << 16, device="cuda").sum()
            assert torch.isfinite(junk)


def test_nothing_to_do(vbq):
    cache = vbq.KVCache(1, 1, 64)
    none = vbq.KVBatch(torch.zeros((0, 1), dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"))
    empty = torch.zeros((0, 1, 64), dtype=torch.float16, device="cuda")
    cache.append(empty, empty, none)
    assert cache.attention(empty, none).shape == (0, 1, 64)
    assert cache.dequant(none)[0].shape == (0, 1, 64)


def test_one_large_value_among_small_ones(vbq):
    """A value scale 2^14 times its neighbours', at every place of a block, equal weights and others."""
    rng = np.random.default_rng(18)
    L = 40
    for factor in (0.0, 1.0):
        for at in range(L):
            c = Case(vbq, rng, [L], 1, 64, kv="f32")
            v = c.v[0].clone()
            v[at] *= 2.0 ** 14
            c.cache.append(c.k[0], v, vbq.KVBatch(c.t, c.l, max_rows=L))
            c.values = [odec.kv_values(_np(v))]
            q = _rows(rng, 1, 2, 64, "f16") * factor
            out = c.cache.attention(q, c.batch([1]), out_dtype=torch.float32)
            _check_attention(out, q, c, [1], 0.125, "f32", what=f"place {at}")


@pytest.mark.parametrize("d,L,rows", [(64, 16450, 130), (128, 8300, 150), (256, 8240, 90)])
def test_parts_that_end_among_a_tiles_rows(vbq, d, L, rows):
    """Split positions whose last part only the later rows of a tile see: every row has its own parts."""
    rng = np.random.default_rng(15 + d)
    _say(f"parts d={d} L={L} rows={rows}")
    c = Case(vbq, rng, [L], 1, d)
    b = c.batch([rows])
    assert c.cache.attention_workspace_size(b, 1) > 0, "this case is meant to split the positions"
    q = torch.zeros((rows, 1, d), dtype=torch.float16, device="cuda")
    out = c.cache.attention(q, b, out_dtype=torch.float32)
    _check_attention(out, q, c, [rows], 0.125, "f32", what=f"parts d={d}")


def test_a_not_finite_position_costs_other_rows_nothing(vbq):
    """Rows that do not see a NaN value keep their precision, small value scales included."""
    rng = np.random.default_rng(16)
    for L, rows, at in ((20, 3, 19), (71, 70, 3), (200, 5, 199)):
        c = Case(vbq, rng, [L], 1, 128, kv="f32")
        k, v = c.k[0].clone(), c.v[0] * 1e-3
        values = odec.kv_values(_np(v))
        v = v.clone()
        v[at, 0, 7] = float("nan")
        c.cache.append(k, v, vbq.KVBatch(c.t, c.l, max_rows=L))
        q = _rows(rng, rows, 2, 128, "f16")
        out = c.cache.attention(q, c.batch([rows]), out_dtype=torch.float32)
        n = at - (L - rows)  # rows that do not see it
        assert torch.isnan(out[n:, :, :64]).all() and torch.isfinite(out[n:, :, 64:]).all()

        class Before:
            hkv, d = 1, 128
        Before.keys, Before.values, Before.lens = [c.keys[0][:at]], [values[:at]], [at]
        _check_attention(out[:n], q[:n], Before, [n], 128 ** -0.5, "f32", what=f"beside NaN, L={L}")


def test_scores_at_the_ends_of_their_range(vbq):
    """Scales and queries at both ends of what is allowed, with hidden positions beside them."""
    rng = np.random.default_rng(17)
    c = Case(vbq, rng, [45], 1, 64)
    q = _rows(rng, 4, 2, 64, "f32")
    for factor, scale in ((2.0 ** -100, 2.0 ** -60), (2.0 ** -60, 2.0 ** 30), (2.0 ** 30, 2.0 ** -40), (0.0, 2.0 ** -60)):
        x = q * factor
        out = c.cache.attention(x, c.batch([4]), scale=scale, out_dtype=torch.float32)
        _check_attention(out, x, c, [4], scale, "f32", what=f"factor {factor} scale {scale}")


def test_calls_on_two_streams_at_once(vbq):
    rng = np.random.default_rng(19)
    c = Case(vbq, rng, [3000, 900, 2000], 2, 128)
    q = [_rows(rng, 3, 8, 128, "f16") for _ in range(2)]
    b = c.batch([1, 1, 1])
    want = [c.cache.attention(x, b) for x in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[c.cache.attention(q[i], b, stream=streams[i]) for i in range(2)] for _ in range(20)]
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o[0], want[0]) and torch.equal(o[1], want[1])


def test_not_finite_queries_stay_in_their_rows(vbq):
    rng = np.random.default_rng(20)
    c = Case(vbq, rng, [90], 1, 128)
    for qt in ("f16", "f32", "bf16"):
        q = _rows(rng, 40, 2, 128, qt)
        want = c.cache.attention(q, c.batch([40]), out_dtype=torch.float32)
        for bad in (float("nan"), float("inf")):
            x = q.clone()
            x[7, 1, 100] = bad
            out = c.cache.attention(x, c.batch([40]), out_dtype=torch.float32)
            assert torch.isnan(out[7, 1]).all()
            out[7, 1], want[7, 1] = 0.0, 0.0
            assert torch.equal(out, want), "rows beside it"
