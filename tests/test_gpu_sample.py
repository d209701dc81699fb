"""The choice of a token against the oracle.

Tokens are whole numbers and have to be equal.  The oracle holds the weights as the same
multiples of 2^-43; its exp and the kernel's may differ in a double's last places, 2^-50 of
a weight at most, which moves a weight by at most one multiple (2^-43) after rounding, so sums
by V 2^-43 of the largest weight.  Where u times the total is nearer than that to a step of
the running sum (or a limit's border to its) either neighbour may be right; the random cases
here keep away from steps (checked), and the ties and borders of the others are exact.
prob is one fp32 rounding of a ratio off by V 2^-43: 2^-24 + 2^-22 allowed.
"""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import decode as odec  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def vbq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2607_02893_amd import vbq as v
    return v


def _dev(a, dtype=np.float32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def _check(vbq, z, u, t=None, k=None, p=None, m=None, near_ok=False, **kw):
    M, V = z.shape
    tok, prob = vbq.sample(z, _dev(u), _dev(t), _dev(k, np.int32), _dev(p), _dev(m), **kw)
    tok, prob = tok.cpu().numpy(), prob.cpu().numpy()
    zn = z.double().cpu().numpy()
    f = lambda a, i, d: d if a is None else float(np.float32(a[i]))  # noqa: E731
    for i in range(M):
        want, share, near = odec.sample(zn[i], f(u, i, 0.5), f(t, i, 1.0), 0 if k is None else int(k[i]), f(p, i, 1.0), f(m, i, 0.0))
        if not near_ok:
            assert near > V * 2.0 ** -43, f"row {i}: a case at a step"
        assert tok[i] == want, f"row {i} V={V}: {tok[i]} instead of {want}"
        assert abs(float(prob[i]) - share) <= (2.0 ** -24 + 2.0 ** -22) * share, f"row {i}"
    return tok


KINDS = ["none", "k", "p", "m", "kp", "km", "pm", "kpm"]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1000, 1025, 4097, 32000, 50257, 128256])
def test_sample_matches_the_oracle(vbq, V, dtype):
    rng = np.random.default_rng(V)
    M = 2 * len(KINDS)
    print(f"sample V={V} {dtype}", flush=True)
    z = torch.from_numpy(3.0 * rng.standard_normal((M, V))).to(TYPES[dtype]).cuda()
    t = rng.uniform(0.4, 1.5, M)
    has = lambda c: np.array([c in KINDS[i % len(KINDS)] and KINDS[i % len(KINDS)] != "none" for i in range(M)])  # noqa: E731
    k = np.where(has("k"), np.exp(rng.uniform(0, np.log(min(V, 5000) + 1), M)).astype(int), 0)
    p = np.where(has("p"), rng.uniform(0.05, 0.99, M), 1.0)
    m = np.where(has("m"), rng.uniform(0.001, 0.4, M), 0.0)
    u = rng.uniform(0, 1, M)
    # fp16 and bf16 logits hold many equal values: the ties' order is tested with them
    _check(vbq, z, u, t, k, p, m)
    _check(vbq, z, u)
    _check(vbq, z, u, t)
    _check(vbq, z, u, None, k)
    _check(vbq, z, u, None, None, p)
    _check(vbq, z, u, t, None, None, m)


@pytest.mark.parametrize("V", [100, 5000, 70001])
def test_every_u_gives_its_token(vbq, V):
    """One row of few candidates at many u: the running sum's order and the ends."""
    rng = np.random.default_rng(V + 1)
    z = np.full(V, -np.inf)
    at = np.sort(rng.choice(V, 9, replace=False))
    z[at] = np.log(np.arange(1, 10))
    M = 90
    u = (np.arange(M) + 0.5) / M
    zt = _dev(np.tile(z, (M, 1)))
    tok = _check(vbq, zt, u)
    assert set(tok) == set(at)
    _check(vbq, zt, u, None, np.full(M, 4))
    _check(vbq, zt, u, None, None, np.full(M, 0.7))
    # the ends: 0 takes the first candidate, numbers up to and past 1 the last
    ends = np.array([0.0, -1.0, np.nan, np.float32(1.0) - 2.0 ** -24, 1.0, 7.0, np.inf])
    got = vbq.sample(zt[:7].contiguous(), _dev(ends))[0].cpu().numpy()
    assert (got[:3] == at[0]).all() and (got[3:] == at[-1]).all()


@pytest.mark.parametrize("V", [40, 3000, 40000])
def test_equal_logits(vbq, V):
    """All logits equal: limits keep the lowest indexes."""
    M = 6
    u = np.array([0.01, 0.3, 0.5, 0.7, 0.9, 0.999])
    for dtype in TYPES.values():
        z = torch.full((M, V), 1.5, dtype=dtype, device="cuda")
        assert np.array_equal(vbq.sample(z, _dev(u))[0].cpu().numpy(), np.floor(np.float64(np.float32(u)) * V))
        for k in (1, 7, V - 1, V, V + 5):
            got = vbq.sample(z, _dev(u), top_k=_dev(np.full(M, k), np.int32))[0].cpu().numpy()
            assert np.array_equal(got, np.floor(np.float64(np.float32(u)) * min(k, V))), k
        got = vbq.sample(z, _dev(u), top_p=_dev(np.full(M, 0.25)))[0].cpu().numpy()
        assert np.array_equal(got, np.floor(np.float64(np.float32(u)) * np.ceil(0.25 * V)))
        got = vbq.sample(z, _dev(u), temperature=_dev(np.zeros(M)))[0].cpu().numpy()
        assert (got == 0).all()
    # two levels, the cut inside the lower one
    z = torch.zeros((M, V), device="cuda")
    z[:, 5::9] = np.log(3.0)
    high = len(range(5, V, 9))
    for k in (high - 1, high, high + 1, high + V // 3):
        if k > 0:
            _check(vbq, z, u, None, np.full(M, k), near_ok=True)
            _check(vbq, z, u, None, np.full(M, k), np.full(M, 0.61803), near_ok=True)


def test_special_rows(vbq):
    inf, nan = np.inf, np.nan
    for V in (16, 4500):
        z = np.tile(np.linspace(-1, 1, V), (12, 1)).astype(np.float32)
        z[0] = nan
        z[1] = -inf
        z[2, 3] = inf
        z[3, [2, 5, V - 1]] = inf
        z[4, ::2] = nan
        z[5, :-1] = -inf
        z[6] = np.finfo(np.float32).min
        z[7] = np.finfo(np.float32).max
        z[8, 0] = 1e38
        z[9] = 0.0
        z[9, 1::2] = -0.0
        z[10] = np.linspace(-3e38, 3e38, V)
        z[11] = np.linspace(-1e-40, 1e-40, V)
        u = np.linspace(0.03, 0.96, 12)
        for t in (1.0, 0.7, 1e-30, 1e30, inf, 0.0, -2.0, nan):
            tok = _check(vbq, _dev(z), u, np.full(12, t), near_ok=True)
            assert tok[0] == -1 and tok[1] == -1 and tok[2] == 3 and tok[5] == V - 1
            _check(vbq, _dev(z), u, np.full(12, t), np.full(12, 3), near_ok=True)
            _check(vbq, _dev(z), u, np.full(12, t), None, np.full(12, 0.4), near_ok=True)
        # limits outside their range
        for k, p, m in ((0, 1.0, 0.0), (-5, 2.0, -1.0), (1, 0.0, 3.0), (2 ** 31 - 1, nan, nan), (2, -1.0, 1.0), (-2 ** 31, inf, inf)):
            _check(vbq, _dev(z), u, None, np.full(12, k), np.full(12, p), np.full(12, m), near_ok=True)


def test_strides_outputs_and_refusals(vbq):
    rng = np.random.default_rng(5)
    wide = _dev(rng.standard_normal((4, 1200)))
    u = rng.uniform(0, 1, 4)
    for lo, V in ((0, 1000), (1, 999), (3, 500)):
        _check(vbq, wide[:, lo:lo + V], u, None, np.array([0, 5, 50, 1]), np.array([0.9, 1.0, 0.3, 0.5]))
    half = wide.half()
    _check(vbq, half[:, 1:1000], u)
    z = wide[:, :64].contiguous()
    tok, prob = torch.full((4,), 9, dtype=torch.int32, device="cuda"), torch.full((4,), 9.0, device="cuda")
    got = vbq.sample(z, _dev(u), tokens=tok, probs=prob)
    assert got[0] is tok and got[1] is prob and vbq.sample(z, _dev(u), probs=False)[1] is None
    assert torch.equal(vbq.sample(z, _dev(u), probs=False)[0], tok)
    for bad in (lambda: vbq.sample(z, _dev(u[:3])), lambda: vbq.sample(z.t(), _dev(u)), lambda: vbq.sample(z.int(), _dev(u)),
                lambda: vbq.sample(z, _dev(u), top_k=_dev(u)), lambda: vbq.sample(z, _dev(u).cpu()), lambda: vbq.sample(z[0], _dev(u)),
                lambda: vbq.sample(z, _dev(u), tokens=tok.long())):
        with pytest.raises(ValueError):
            bad()
    assert vbq.sample(torch.empty((0, 64), device="cuda"), _dev(u[:0]))[0].shape == (0,)


def test_many_rows_and_the_largest_vocabulary(vbq):
    rng = np.random.default_rng(6)
    z = _dev(rng.standard_normal((300, 777)))
    _check(vbq, z, rng.uniform(0, 1, 300), None, rng.integers(0, 100, 300), rng.uniform(0.1, 1.2, 300))
    z = _dev(2.0 * rng.standard_normal((2, 1 << 20)))
    _check(vbq, z, np.array([0.41, 0.83]))
    _check(vbq, z, np.array([0.41, 0.83]), None, np.array([30000, 0]), np.array([0.95, 0.9]))


def test_streams_and_graphs(vbq):
    rng = np.random.default_rng(7)
    M, V = 5, 33333
    z, u = _dev(3 * rng.standard_normal((M, V))), _dev(rng.uniform(0, 1, M))
    k, p = _dev(np.array([0, 40, 0, 3000, 1]), np.int32), _dev(np.array([0.9, 0.9, 1.0, 1.0, 0.2]))
    want = vbq.sample(z, u, None, k, p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = vbq.sample(z, u, None, k, p, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    ws = torch.empty(max(16, vbq.sample_workspace_size(M, V)), dtype=torch.uint8, device="cuda")
    toks = [torch.empty(M, dtype=torch.int32, device="cuda") for _ in range(2)]
    zs = [z, _dev(3 * rng.standard_normal((M, V)))]
    graphs = []
    for i in range(2):  # two graphs on one workspace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            vbq.sample(zs[i], u, None, k, p, tokens=toks[i], probs=False, workspace=ws)
        graphs.append(g)
    for step in range(4):
        u.copy_(_dev(rng.uniform(0, 1, M)))
        for i in range(2):
            toks[i].fill_(-7)
            ws.fill_(0xAB)   # what a workspace held before does not matter
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(toks[i], vbq.sample(zs[i], u, None, k, p)[0]), (step, i)


def test_more_rows_than_are_taken_at_once(vbq):
    """Long rows come in sets that share the workspace, one after the other."""
    rng = np.random.default_rng(8)
    z = _dev(3 * rng.standard_normal((150, 4500)))
    _check(vbq, z, rng.uniform(0, 1, 150), rng.uniform(0.5, 1.4, 150), rng.integers(0, 300, 150), rng.uniform(0.3, 1.1, 150))


def test_calls_on_two_streams_at_once(vbq):
    rng = np.random.default_rng(9)
    z = [_dev(3 * rng.standard_normal((4, 20000))) for _ in range(2)]
    u, k, p = _dev(rng.uniform(0, 1, 4)), _dev(np.array([0, 40, 0, 300]), np.int32), _dev(np.array([0.9, 0.8, 1.0, 1.0]))
    want = [vbq.sample(x, u, None, k, p)[0] for x in z]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[vbq.sample(z[i], u, None, k, p, stream=streams[i])[0] for i in range(2)] for _ in range(20)]
    torch.cuda.synchronize()
    for g in got:
        assert torch.equal(g[0], want[0]) and torch.equal(g[1], want[1])
