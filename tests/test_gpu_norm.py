"""Residual sum and norm against the oracle.

h is exact: one fp32 sum, one rounding.  x, with u = 2^-24: a lane adds at most K/256 + 8
squares in a row and the tree adds 8 levels, each rounding u, so the mean is off by at most
(K/256 + 18) u relative and its root by half of that; the root, the reciprocal and the two
products add 4 roundings, and the output's type half a step (2^-11 fp16, 2^-8 bf16, 2^-24 fp32).
Below fp16's normals a step is 2^-24, half of it 2^-25.
"""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import decode as odec  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-38, "f16": 2.0 ** -25, "bf16": 1e-38}


@pytest.fixture(scope="module")
def vbq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2607_02893_amd import vbq as v
    return v


def _np(t):
    return t.double().cpu().numpy()


def _rand(rng, shape, dtype, scale=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(TYPES[dtype]).cuda()


def _check(x, h, residual, y, weight, eps, res_type, x_type):
    K = residual.shape[-1]
    want, hw = odec.add_norm(_np(residual), None if y is None else _np(y), None if weight is None else _np(weight), eps, res_type)
    if h is not None:
        assert np.array_equal(_np(h), hw)
    bound = np.abs(want) * (((K / 256 + 18) / 2 + 4) * 2.0 ** -24 + HALF_STEP[x_type]) + TINY[x_type]
    err = np.abs(_np(x) - want)
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("res,yt,xt", [("f16", "f32", "f16"), ("bf16", "bf16", "bf16"), ("f32", "f16", "f16"), ("f32", "f32", "f32"),
                                       ("bf16", "f32", "f16")])
@pytest.mark.parametrize("m,K", [(1, 1), (3, 7), (2, 64), (5, 100), (1, 2048), (2, 4095), (2, 4096), (1, 8192), (1, 8200), (2, 8201),
                                 (1, 16384), (1, 50001), (700, 128), (33, 5120)])
def test_norm_matches_the_oracle(vbq, m, K, res, yt, xt):
    print(f"norm m={m} K={K} {res}+{yt}->{xt}", flush=True)
    rng = np.random.default_rng(K + m)
    residual, y = _rand(rng, (m, K), res, 3.0), _rand(rng, (m, K), yt)
    weight = _rand(rng, (K,), xt)
    x, h = vbq.add_norm(residual, y, weight, 1e-5, x_dtype=TYPES[xt])
    _check(x, h, residual, y, weight, 1e-5, res, xt)
    # in place: the residual becomes the sum
    r2 = residual.clone()
    x2, h2 = vbq.add_norm(r2, y, weight, 1e-5, h=r2, x_dtype=TYPES[xt])
    assert h2 is r2 and torch.equal(r2, h) and torch.equal(x2, x)
    # without y, without weight, without h
    x3, h3 = vbq.add_norm(h, None, weight, 1e-5, x_dtype=TYPES[xt])
    assert torch.equal(x3, x) and h3 is h
    x4, h4 = vbq.add_norm(residual, y, None, 1e-3, h=False, x_dtype=TYPES[xt])
    assert h4 is None
    _check(x4, None, residual, y, None, 1e-3, res, xt)


def test_norm_strides_alignment_and_dimensions(vbq):
    rng = np.random.default_rng(1)
    wide = _rand(rng, (6, 300), "f32")
    for lo, K in ((0, 256), (4, 256), (1, 256), (8, 255), (3, 7)):
        residual, y = wide[:, lo:lo + K], _rand(rng, (6, K), "f16")
        out = torch.full((6, 320), 5.0, dtype=torch.float16, device="cuda")
        x = out[:, lo:lo + K]
        _, h = vbq.add_norm(residual, y, None, 1e-6, x=x)
        _check(x, h, residual, y, None, 1e-6, "f32", "f16")
        assert (out[:, :lo] == 5.0).all() and (out[:, lo + K:] == 5.0).all()
    # a broadcast y: rows that share memory are read as they are
    one = _rand(rng, (1, 64), "f32")
    with pytest.raises(vbq.VbqError):
        vbq.add_norm(wide[:, :64], one.expand(6, 64))
    r3 = _rand(rng, (2, 3, 64), "bf16")
    x, h = vbq.add_norm(r3, r3, None, 1e-6)
    assert x.shape == r3.shape and x.dtype == torch.float16
    _check(x.reshape(6, 64), h.reshape(6, 64), r3.reshape(6, 64), r3.reshape(6, 64), None, 1e-6, "bf16", "f16")
    for bad in (lambda: vbq.add_norm(r3, r3[:1]), lambda: vbq.add_norm(r3, r3, r3[0, 0][:32]), lambda: vbq.add_norm(r3, r3.cpu()),
                lambda: vbq.add_norm(r3, r3, h=r3.half()), lambda: vbq.add_norm(r3.transpose(0, 1), r3.transpose(0, 1)),
                lambda: vbq.add_norm(r3.int(), r3), lambda: vbq.add_norm(r3, r3, x=torch.empty(64, device="cuda").expand(2, 3, 64))):
        with pytest.raises(ValueError):
            bad()
    assert vbq.add_norm(torch.empty((0, 64), device="cuda"))[0].shape == (0, 64)


def test_norm_edges(vbq):
    # zeros with eps, and rows that are not finite, which stay by themselves
    z = torch.zeros((4, 128), device="cuda")
    x, _ = vbq.add_norm(z, None, None, 1e-6, x_dtype=torch.float32)
    assert (x == 0).all()
    x, _ = vbq.add_norm(z, None, None, 0.0, x_dtype=torch.float32)
    assert torch.isnan(x).all()          # 0 / 0
    r = torch.ones((3, 128), device="cuda")
    r[1, 5] = float("nan")
    x, h = vbq.add_norm(r, r, None, 1e-6, x_dtype=torch.float32)
    assert torch.isnan(x[1]).all() and torch.isfinite(x[[0, 2]]).all() and torch.isnan(h[1, 5])
    # an fp16 stream that overflows holds infinity, as its type does
    r = torch.full((1, 64), 60000.0, dtype=torch.float16, device="cuda")
    _, h = vbq.add_norm(r, r)
    assert torch.isinf(h).all()


def test_norm_streams_and_graphs(vbq):
    rng = np.random.default_rng(2)
    r, y, w = _rand(rng, (5, 1024), "f16"), _rand(rng, (5, 1024), "f32"), _rand(rng, (1024,), "f32")
    want, hw = vbq.add_norm(r, y, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    x, h = vbq.add_norm(r, y, w, stream=side)
    side.synchronize()
    assert torch.equal(x, want) and torch.equal(h, hw)
    g = torch.cuda.CUDAGraph()
    x, h = torch.empty_like(want), torch.empty_like(hw)
    with torch.cuda.graph(g):
        vbq.add_norm(r, y, w, x=x, h=h)
    for i in range(3):
        r.copy_(_rand(rng, (5, 1024), "f16"))
        g.replay()
        torch.cuda.synchronize()
        want, hw = vbq.add_norm(r, y, w)
        assert torch.equal(x, want) and torch.equal(h, hw), i
