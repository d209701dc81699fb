"""More rows than one launch takes: a grid dimension holds fewer than 2^32 threads, which a
workgroup a row reaches at 2^24 rows."""

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vbq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    from paper_2607_02893_amd import vbq as v
    return v


@pytest.mark.parametrize("n,pad", [((1 << 24) + 3, 0), ((1 << 22) + 1, 8)])
def test_norm_of_many_rows(vbq, n, pad):
    """Rows that repeat give results that repeat, to the last row; padding stays as it was."""
    print(f"norm n={n} pad={pad}", flush=True)
    K, period = 8, 200
    gen = torch.Generator(device="cuda").manual_seed(1)
    few = torch.randn((period, K), generator=gen, device="cuda").half()
    y = torch.randn((period, K), generator=gen, device="cuda")
    weight = torch.randn(K, generator=gen, device="cuda")
    want, hw = vbq.add_norm(few, y, weight)
    row = torch.arange(n, device="cuda") % period
    many = few[row]
    x = torch.full((n, K + pad), 3.0, dtype=torch.float16, device="cuda")
    _, h = vbq.add_norm(many, y[row], weight, x=x[:, :K])
    assert torch.equal(x[:, :K], want[row]) and torch.equal(h, hw[row])
    assert (x[:, K:] == 3.0).all()
    vbq.add_norm(many, y[row], weight, h=many, x=x[:, :K])
    assert torch.equal(many, hw[row]) and torch.equal(x[:, :K], want[row])
