"""Operators on token tables and class scores where values, weights and sizes are at their limits, through every kernel that sizes choose.

The definitions in 64 bits, the units and the bounds are those of test_gpu_head.py."""
import math

import pytest
import torch

from test_gpu_head import ROUND, U, _close, _definition, _gen, _problem, ctx  # noqa: F401

pytestmark = pytest.mark.gpu

# rows, values, classes: few rows, short rows that are swept, tiles (both products at once, and one after the other)
BF16_SHAPES = [(3, 40, 500), (9, 264, 3000), (16, 512, 130), (60, 64, 500), (200, 128, 700), (333, 250, 900), (33, 300, 200), (300, 520, 1000), (2100, 264, 2300)]


def _gradients_fit(x, w, u, got, gx, gw, smag, pu, d, lse):
    """The bound of test_softmax_loss_and_gradients on both gradients (None: not looked at)."""
    dtype = x.dtype
    serr = 32 * U * smag.amax(1)
    perr = (2 * serr + 64 * U * (2 + smag.amax(1) + lse.abs())).unsqueeze(1) * pu
    e = perr + ((2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23) + 32 * U) * d.abs()
    r = ROUND[dtype]
    if got[0] is not None:
        assert bool(((got[0].cpu().double() - gx).abs() <= r * gx.abs() + e @ w.double().abs() + 1e-30).all())
    if got[1] is not None:
        assert bool(((got[1].cpu().double() - gw).abs() <= r * gw.abs() + e.t() @ x.double().abs() + 1e-30).all())


@pytest.mark.parametrize("n,dim,vocab", BF16_SHAPES)
def test_left_out_rows_and_a_class_of_infinite_weights(ctx, n, dim, vocab):  # noqa: F811
    """A class whose weights are -infinity has a score of -infinity in every live row (all x are positive) and D = 0: its gradient is zero and the others'
    are those without it, however many rows are left out and whatever these hold."""
    x, w, t, u = _problem(n, dim, vocab, torch.bfloat16)
    x = (x.float().abs() + 0.125).bfloat16()
    t = torch.where(t == 3, 4, t)
    t[0], u[0] = 5, 0.0
    t[1] = -1
    w = (w.float() * 0.25).bfloat16()
    masked = w.clone()
    masked[3] = float("-inf")
    rest = torch.cat([w[:3], w[4:]])
    loss, lse, gx, gw, smag, pu, d, ok = _definition(x, rest, torch.where(t > 3, t - 1, t), u)
    bad = x.clone()
    bad[1] = float("nan")
    got_loss, got_lse = ctx.softmax_loss(bad.cuda(), masked.cuda(), t.cuda())
    gw_got = ctx.softmax_gradients(bad.cuda(), masked.cuda(), t.cuda(), got_lse, u.cuda(), need_x=False)[1]
    assert bool(torch.isfinite(gw_got).all()) and bool((gw_got[3] == 0).all())
    _gradients_fit(x, rest, u, (None, torch.cat([gw_got[:3], gw_got[4:]])), gx, gw, smag, pu, d, lse)
    # both at once: the class weights' gradient is the same
    assert torch.equal(ctx.softmax_gradients(bad.cuda(), masked.cuda(), t.cuda(), got_lse, u.cuda())[1], gw_got)


# fp32: few rows; swept; weights where they lie; both second products at once; tiles
F32_SHAPES = [(3, 40, 500), (16, 512, 130), (60, 64, 500), (200, 100, 700), (1500, 40, 300), (100, 192, 3000), (300, 520, 1000), (130, 200, 1000), (2100, 264, 2300)]
SHAPES = [(torch.bfloat16,) + s for s in BF16_SHAPES + [(1500, 40, 300)]] + [(torch.float32,) + s for s in F32_SHAPES]


@pytest.mark.parametrize("dtype,n,dim,vocab", SHAPES)
def test_weights_of_very_different_size(ctx, dtype, n, dim, vocab):  # noqa: F811
    """Row weights over 27 orders of magnitude, the first one that counts 39 below the largest: gradients as by the definition."""
    x, w, t, u = _problem(n, dim, vocab, dtype)
    g = _gen(n)
    u = torch.where(u > 0, 10.0 ** (27.0 * torch.rand(n, generator=g, dtype=torch.float64) - 18.0), 0.0).float()
    t[0], u[0] = 1, 2e-30
    t[n - 1], u[n - 1] = 2, 1e9
    loss, lse, gx, gw, smag, pu, d, ok = _definition(x, w, t, u)
    got_lse = ctx.softmax_loss(x.cuda(), w.cuda(), t.cuda())[1]
    for sign in (1.0, -1.0):
        got = ctx.softmax_gradients(x.cuda(), w.cuda(), t.cuda(), got_lse, sign * u.cuda())
        _gradients_fit(x, w, u, got, sign * gx, sign * gw, smag, pu, d, lse)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [40, 264])
def test_the_rows_that_count_come_last(ctx, dtype, dim):  # noqa: F811
    """Thousands of rows without target, then some with: the gradients as of these alone."""
    n, live, vocab = 140_000, 500, 300
    x, w, t, u = _problem(live, dim, vocab, dtype)
    t = t % vocab
    pad = torch.zeros(n - live, dim, dtype=dtype)
    none, one = torch.full((n - live,), -1), torch.ones(n - live)
    lse = ctx.softmax_loss(x.cuda(), w.cuda(), t.cuda())[1].cpu()
    last = [torch.cat(a).cuda() for a in ((pad, x), (none, t), (one * 0, lse), (one, u))]
    got = ctx.softmax_gradients(last[0], w.cuda(), last[1], last[2], last[3])
    _, want_lse, gx, gw, smag, pu, d, ok = _definition(x, w, t, u)
    assert bool((got[0][:n - live] == 0).all())
    _gradients_fit(x, w, u, (got[0][n - live:], got[1]), gx, gw, smag, pu, d, want_lse)
