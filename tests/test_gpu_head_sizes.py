"""Operators on token tables and class scores at the largest sizes that they accept: counts next to 2^31, launches next to 2^32 threads."""
import math

import pytest
import torch

from test_gpu_head import U, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def _needs(gigabytes):
    if torch.cuda.mem_get_info()[0] < gigabytes * 1e9:
        pytest.skip(f"needs {gigabytes} GB of device memory")


def _parts(n):
    return [(a, min(n, a + 2 ** 28)) for a in range(0, n, 2 ** 28)]


def test_softmax_of_as_many_rows_as_there_may_be(ctx):  # noqa: F811
    _needs(140)
    n = MOST
    at = torch.tensor([0, 5, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 301, n - 200, n - 64, n - 63, n - 2, n - 1], device="cuda")
    x = torch.zeros(n, 1, dtype=torch.bfloat16, device="cuda")
    t = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    u = torch.zeros(n, device="cuda")
    x[at], t[at], u[at] = 1.0, 0, 0.5
    w = torch.tensor([[0.5], [0.0]], dtype=torch.bfloat16, device="cuda")
    loss, lse = ctx.softmax_loss(x, w, t)
    one = math.log(math.exp(0.5) + 1.0)
    assert bool(((lse[at].double() - one).abs() <= 32 * U).all()) and bool(((loss[at].double() - (one - 0.5)).abs() <= 32 * U).all())
    lse[at] = math.log(2.0)
    for a, b in _parts(n):
        assert float((lse[a:b] - math.log(2.0)).abs().max()) <= 32 * U
    lse[at] = one
    del loss
    gx, gw = ctx.softmax_gradients(x, w, t, lse, u)
    p = 1.0 / (1.0 + math.exp(-0.5))
    # D is rounded to bfloat16, and so are the results
    assert bool(((gx[at, 0].double() - 0.5 * (p - 1.0) * 0.5).abs() <= 0.25 * 2.0 ** -7).all())
    assert sum(int((gx[a:b] != 0).sum()) for a, b in _parts(n)) == len(at)
    assert abs(float(gw[0]) - 5.0 * (p - 1.0)) <= 5.0 * 2.0 ** -7 and abs(float(gw[1]) - 5.0 * (1.0 - p)) <= 5.0 * 2.0 ** -7


def test_lookup_gradient_of_as_many_tokens_as_there_may_be(ctx):  # noqa: F811
    """One token in all places but a few: its entries end with the last one, 2^31 - 1."""
    _needs(80)
    n = MOST
    t = torch.ones(n, dtype=torch.int32, device="cuda")
    grad = torch.zeros(n, 1, dtype=torch.bfloat16, device="cuda")
    t[3], t[n - 9], grad[3], grad[n - 9] = 0, 0, 3.0, 4.0
    at = torch.tensor([0, 1, 17, 2 ** 30, 2 ** 31 - 70, n - 8, n - 7, n - 2, n - 1], device="cuda")
    grad[at] = 1.0
    got = ctx.embed_gradient(t, grad, 3)
    assert got[:, 0].tolist() == [7.0, 9.0, 0.0]


def test_lookup_gradient_of_many_entries_of_wide_rows(ctx):  # noqa: F811
    """A workgroup per token and sixteen entries of each would be 2^32 threads: few rows of 1024 values in very large bags."""
    _needs(20)
    n, bag, dim, vocab = 4200, 65536, 1024, 4096
    t = torch.randint(0, vocab, (n, bag), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    grad = (torch.arange(n, device="cuda") % 8 == 0).float()[:, None] * (1.0 + torch.arange(dim, device="cuda").float()[None]) / 1024.0
    counts = torch.zeros(n, vocab, dtype=torch.float64, device="cuda")
    for a in range(0, n, 300):
        rows = t[a:a + 300].long()
        counts[a:a + 300].scatter_add_(1, rows, torch.ones(rows.shape, dtype=torch.float64, device="cuda"))
    got = ctx.embed_gradient(t, grad, vocab + 1)
    want = counts.t().contiguous() @ grad.double()
    assert bool(((got[:vocab].double() - want).abs() <= 33 * U * want).all())
    assert bool((got[vocab] == 0).all())


def test_loss_of_many_rows_against_millions_of_classes(ctx):  # noqa: F811
    """131,072 rows at once against so many classes would be 2^32 threads of the largest tiles: the rows are taken in smaller blocks."""
    _needs(30)
    n, dim, vocab = 131_072 + 5, 264, 4_400_003
    g = torch.Generator(device="cuda").manual_seed(2)
    w = torch.randn(vocab, dim, generator=g, device="cuda", dtype=torch.bfloat16) * 0.06
    t = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    x = torch.randn(n, dim, generator=g, device="cuda", dtype=torch.bfloat16)
    loss, lse = ctx.softmax_loss(x, w, t)
    at = torch.tensor([0, 1, 16383, 16384, 32767, 32768, 65535, 65536, 131_071, 131_072, n - 1], device="cuda")
    want = torch.full((len(at),), -math.inf, dtype=torch.float64, device="cuda")
    mag = torch.zeros(len(at), dtype=torch.float64, device="cuda")
    for a in range(0, vocab, 200_000):
        ws = w[a:a + 200_000].double()
        want = torch.logaddexp(want, torch.logsumexp(x[at].double() @ ws.t(), 1))
        mag = torch.maximum(mag, (x[at].double().abs() @ ws.abs().t()).amax(1))
    score = (x[at].double() * w[t[at]].double()).sum(1)
    assert bool(((lse[at].double() - want).abs() <= 32 * U * (1 + mag + want.abs())).all())
    assert bool(((loss[at].double() - (want - score)).abs() <= 64 * U * (1 + mag + want.abs())).all())
    assert bool(torch.isfinite(loss).all())
