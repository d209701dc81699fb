"""A decode layer as a serving loop runs it, every stage through the library: norm, the
packed Q|K|V product, append, attention, the packed O product, residual norm, the packed
head, the choice of a token.  Each stage is checked on what the stage before it gave, with
that stage's own bound, for prompts of several rows first and then token by token."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import decode as odec  # noqa: E402
from oracle import matmul as omatmul  # noqa: E402
from paper_2607_02893_amd import synth  # noqa: E402
from tests import parity  # noqa: E402
from tests.test_gpu_cache import _check_attention  # noqa: E402
from tests.test_gpu_norm import _check as _check_norm  # noqa: E402

pytestmark = pytest.mark.gpu

D, HQ, HKV, HD, V = 512, 8, 2, 64, 4000


@pytest.fixture(scope="module")
def vbq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2607_02893_amd import vbq as v
    return v


class Packed:
    def __init__(self, vbq, rng, N, K):
        bits = synth.draw_bits(rng, N, K // 64, synth.MIX_PILOT)
        self.q, self.s = synth.draw_levels(rng, bits), synth.draw_scales(rng, N, K // 64)
        self.m = vbq.PackedMatrix(*vbq.pack_codes(self.q, self.s, bits))

    def __call__(self, x):
        Y = self.m.gemm_small(x)
        xn = x.cpu().numpy()
        for i in range(x.shape[0]):
            parity.check(Y[i].cpu().numpy(), omatmul.gemv(self.q, self.s, xn[i]), omatmul.row_magnitude(self.q, self.s, xn[i]), what="product")
        return Y


def test_a_decode_layer(vbq):
    rng = synth.rng_for(77)
    nrng = np.random.default_rng(77)
    qkv, o, head = Packed(vbq, rng, (HQ + 2 * HKV) * HD, D), Packed(vbq, rng, D, HQ * HD), Packed(vbq, rng, V, D)
    w1, w2 = [torch.from_numpy(1 + 0.1 * nrng.standard_normal(D)).float().cuda() for _ in range(2)]
    embed = torch.from_numpy(nrng.standard_normal((V, D))).half().cuda()
    n = 3
    cache = vbq.KVCache(8, HKV, HD)
    table = torch.tensor([[5, 2], [0, 7], [3, 1]], dtype=torch.int32, device="cuda")
    lens = torch.zeros(n, dtype=torch.int32, device="cuda")
    held = [[[], []] for _ in range(n)]

    class C:
        pass

    def step(rows, tokens):
        """rows[b] tokens of each sequence; returns the tokens chosen after the last rows."""
        starts = np.concatenate([[0], np.cumsum(rows)])
        total = int(starts[-1])
        lens.add_(torch.tensor(rows, dtype=torch.int32, device="cuda"))
        batch = vbq.KVBatch(table, lens, torch.tensor(starts, dtype=torch.int32, device="cuda"), n_rows=total, max_rows=max(rows))
        stream = embed[tokens]
        x, _ = vbq.add_norm(stream, None, w1, 1e-5)
        _check_norm(x, None, stream, None, w1, 1e-5, "f16", "f16")
        y = qkv(x).unflatten(1, (HQ + 2 * HKV, HD))
        q, k, v = y[:, :HQ], y[:, HQ:HQ + HKV], y[:, HQ + HKV:]
        cache.append(k, v, batch)
        for b in range(n):
            for i, t in enumerate((k, v)):
                held[b][i].extend(odec.kv_values(t[starts[b]:starts[b + 1]].double().cpu().numpy()))
        a = cache.attention(q, batch, out_dtype=torch.float16)
        c = C()
        c.keys, c.values = [np.array(h[0]) for h in held], [np.array(h[1]) for h in held]
        c.lens, c.hkv, c.d = [len(h[0]) for h in held], HKV, HD
        _check_attention(a, q, c, rows, HD ** -0.5, "f16", what=f"step {rows}")
        z = o(a.flatten(1))
        x, h = vbq.add_norm(stream, z, w2, 1e-5)
        _check_norm(x, h, stream, z, w2, 1e-5, "f16", "f16")
        last = x[torch.tensor(starts[1:] - 1, device="cuda")].contiguous()
        logits = head(last)
        u = torch.from_numpy(nrng.uniform(0, 1, n)).float().cuda()
        t = torch.tensor([1.0, 20.0, 0.0], device="cuda")
        kk, p = torch.tensor([0, 40, 5], dtype=torch.int32, device="cuda"), torch.tensor([0.9, 0.95, 1.0], device="cuda")
        tok, _ = vbq.sample(logits, u, t, kk, p)
        for b in range(n):
            want, _, near = odec.sample(logits[b].double().cpu().numpy(), float(u[b]), float(t[b]), int(kk[b]), float(p[b]))
            assert near > V * 2.0 ** -43 and int(tok[b]) == want
        return tok.long()

    tokens = torch.from_numpy(nrng.integers(0, V, 16)).cuda()
    nxt = step([7, 1, 8], tokens)
    for _ in range(4):
        nxt = step([1, 1, 1], nxt)
