"""Operators on token tables and class scores where values, weights and sizes are at their limits, through every kernel that sizes choose.

The definitions in 64 bits, the units and the bounds are those of test_gpu_head.py."""
import math

import pytest
import torch

from test_gpu_head import ROUND, U, _definition, _gen, _problem, ctx  # noqa: F401
from test_head_pieces import coherent

pytestmark = pytest.mark.gpu

# rows, values, classes: few rows, short rows that are swept, tiles (both products at once, and one after the other)
BF16_SHAPES = [(3, 40, 500), (9, 264, 3000), (16, 512, 130), (60, 64, 500), (200, 128, 700), (333, 250, 900), (33, 300, 200), (300, 520, 1000), (2100, 264, 2300)]


def _gradients_fit(x, w, u, got, gx, gw, smag, pu, d, lse):
    """The bound of test_softmax_loss_and_gradients on both gradients (None: not looked at), and for what fp32 cannot hold of D in units of the largest weight: below 2^-126
    it may hold nothing."""
    dtype = x.dtype
    serr = 32 * U * smag.amax(1)
    perr = (2 * serr + 64 * U * (2 + smag.amax(1) + lse.abs())).unsqueeze(1) * pu
    e = perr + ((2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23) + 32 * U) * d.abs() + 2.0 ** -126 * float(u.abs().max())
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


# ---- fp32 scores of rows whose values differ much in size ------------------------------------------------


def _uneven(n, dim, vocab, kind):
    """fp32 rows whose scores are sums of terms of one size, or of few terms, while the rows themselves range over many orders of magnitude."""
    x, w, t, u = _problem(n, dim, vocab, torch.float32)
    g = _gen(n + dim)
    if kind == "one column":  # 1e8 times larger in x and as much smaller in the weights
        x[:, 3] *= 1e8
        w[:, 3] *= 1e-8
    elif kind == "columns":  # powers of ten from -15 to 15
        f = 10.0 ** (30.0 * torch.rand(dim, generator=g, dtype=torch.float64) - 15.0)
        x, w = (x.double() * f).float(), (w.double() / f).float()
    elif kind == "rows of their own":  # each row has its large value where the weights are small
        at = torch.randint(0, dim // 4, (n,), generator=g)
        x[torch.arange(n), at] *= 1e9
        w[:, :dim // 4] *= 1e-9
    elif kind == "one value":  # of each row of x, which meets a small value of every class
        at = torch.randint(0, dim - 1, (n,), generator=g)
        x = torch.zeros_like(x)
        x[torch.arange(n), at] = 1e10 * torch.rand(n, generator=g)
        w[:, dim - 1] *= 1e10
        w *= 1e-10
    elif kind == "wide":  # scores of 1e4, which scaled back by one of the rows' powers of two alone are beyond fp32
        x, w = x * 1e37, w * 1e-33
    return x, w, t, u


UNEVEN = ["one column", "columns", "rows of their own", "one value", "wide"]
UNEVEN_SHAPES = [(16, 72, 300), (40, 512, 130), (60, 64, 500), (200, 100, 700), (3000, 128, 300), (100, 192, 3000), (300, 520, 1000), (600, 136, 8300), (2100, 264, 2300), (1300, 1032, 3000)]


@pytest.mark.parametrize("kind", UNEVEN)
@pytest.mark.parametrize("n,dim,vocab", UNEVEN_SHAPES)
def test_fp32_scores_of_uneven_rows(ctx, n, dim, vocab, kind):  # noqa: F811
    """The bounds of test_softmax_loss_and_gradients, which go by the sum of a score's magnitudes, whatever the rows' own range is."""
    x, w, t, u = _uneven(n, dim, vocab, kind)
    loss, lse, gx, gw, smag, pu, d, ok = _definition(x, w, t, u)
    got_loss, got_lse = ctx.softmax_loss(x.cuda(), w.cuda(), t.cuda())
    serr = 32 * U * smag.amax(1)
    assert bool(((got_lse.cpu().double() - lse).abs() <= serr + 32 * U * (1 + lse.abs())).all())
    assert bool(((got_loss.cpu().double() - loss).abs() <= 2 * serr + 32 * U * (1 + lse.abs() + smag.amax(1))).all())
    _gradients_fit(x, w, u, ctx.softmax_gradients(x.cuda(), w.cuda(), t.cuda(), got_lse, u.cuda()), gx, gw, smag, pu, d, lse)


@pytest.mark.parametrize("n,dim,vocab,at", [(131_200, 132, 20, 131_150), (131_200, 132, 20, 7), (300_000, 40, 24, 290_000)])
def test_one_uneven_row_among_blocks_of_rows(ctx, n, dim, vocab, at):  # noqa: F811
    """Of rows that are taken in blocks, one in the last block, or in the first, asks for other pieces than the rest."""
    x, w, t, u = _problem(n, dim, vocab, torch.float32)
    w[:, 2] *= 1e-9
    x[at] *= 0.25
    x[at, 2] = 3e8
    got_loss, got_lse = (a.cpu().double() for a in ctx.softmax_loss(x.cuda(), w.cuda(), t.cuda()))
    some = torch.cat([torch.arange(100), torch.arange(at - 7, at + 50), torch.arange(n - 50, n)])
    loss, lse, gx, gw, smag, pu, d, ok = _definition(x[some], w, t[some], u[some])
    serr = 32 * U * smag.amax(1)
    assert bool(((got_lse[some] - lse).abs() <= serr + 32 * U * (1 + lse.abs())).all())
    assert bool(((got_loss[some] - loss).abs() <= 2 * serr + 32 * U * (1 + lse.abs() + smag.amax(1))).all())
    g = ctx.softmax_gradients(x.cuda(), w.cuda(), t.cuda(), got_lse.float().cuda(), u.cuda())
    _gradients_fit(x[some], w, u[some], (g[0].cpu()[some], None), gx, gw, smag, pu, d, lse)


@pytest.mark.parametrize("kind", ["even", "one column"])
@pytest.mark.parametrize("n,dim,vocab", [(16, 72, 2), (60, 64, 2), (200, 128, 2), (100, 192, 2), (2500, 264, 520), (70_000, 136, 24)])
def test_no_piece_of_fp32_values_is_lost(ctx, n, dim, vocab, kind):  # noqa: F811
    """Values whose products of pieces add up, so that one that is left out, or taken twice, shows (test_head_pieces.py has what each would do).  Two classes have positive scores,
    and the gradients' sums few large terms.  Bounds: 16 u of the sum of magnitudes for a score, for a gradient what that makes of p and 8 u of its own."""
    x, w = coherent(n, dim, 1), coherent(vocab, dim, 2)
    w[2:] = -w[2:]
    if kind == "one column":
        x[:, 5] *= 2.0 ** 26
        w[:, 5] *= 2.0 ** -26
        x[:, 6] *= 2.0 ** -26
        w[:, 6] *= 2.0 ** 26
    t, u = torch.arange(n) % 2, torch.ones(n)
    loss, lse, gx, gw, smag, pu, d, ok = _definition(x, w, t, u)
    got_loss, got_lse = ctx.softmax_loss(x.cuda(), w.cuda(), t.cuda())
    top = smag[:, :2].amax(1)
    assert bool(((got_lse.cpu().double() - lse).abs() <= 16 * U * (top + 1)).all())
    got = ctx.softmax_gradients(x.cuda(), w.cuda(), t.cuda(), got_lse, u.cuda())
    # p (1 - p) at most 1/4 times the error of s - lse, both classes
    perr = 32 * U * (top + 1)[:, None] * (pu * (1 - pu) + 1e-12) + 8 * U * d.abs()
    assert bool(((got[0].cpu().double() - gx).abs() <= perr @ w.double().abs() + 8 * U * (d.abs() @ w.double().abs()) + 1e-30).all())
    assert bool(((got[1].cpu().double() - gw).abs() <= perr.t() @ x.double().abs() + 8 * U * (d.abs().t() @ x.double().abs()) + 1e-30).all())


@pytest.mark.parametrize("where", ["x", "weight"])
@pytest.mark.parametrize("n,dim,vocab", [(16, 72, 300), (60, 64, 500), (200, 100, 700), (100, 192, 3000), (600, 136, 8300), (2100, 264, 2300)])
def test_infinite_fp32_values_make_scores_that_are_no_numbers(ctx, n, dim, vocab, where):  # noqa: F811
    """An infinity that meets values of one sign, in all of their pieces: the header says NaN, and not -infinity, which adds nothing."""
    x, w, t, u = _problem(n, dim, vocab, torch.float32)
    w[:, 3] = -(1.0 + 2.0 ** -10 + 2.0 ** -20)
    x[:, 3] = 1.0 + 2.0 ** -10 + 2.0 ** -20
    base = ctx.softmax_loss(x.cuda(), w.cuda(), t.cuda())[1].cpu()
    if where == "x":
        x[7, 3] = float("inf")
    else:
        w[11, 3] = float("-inf")
    for again in (False, True):  # (and where another row asks for more pieces)
        lse = ctx.softmax_loss(x.cuda(), w.cuda(), t.cuda())[1].cpu()
        if where == "x":
            assert bool(torch.isnan(lse[7])) and bool(torch.isfinite(torch.cat([lse[:7], lse[8:]])).all())
            assert again or torch.equal(torch.cat([lse[:7], lse[8:]]), torch.cat([base[:7], base[8:]]))
        else:
            assert bool(torch.isnan(lse).all())
        x[9] *= 1e-12
        x[9, 1] = 1.0


# ---- long sums -----------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,bag,dim,vocab", [(3, 60_000, 12, 500), (2, 65_536, 33, 1), (5, 40_001, 3, 2), (70, 3001, 260, 3)])
def test_lookup_of_long_bags(ctx, dtype, n, bag, dim, vocab):  # noqa: F811
    """Few distinct values, added up tens of thousands of times: the roundings of a sum of one after the other would all go one way.  Sums of eight and a sum of these
    that keeps its roundings are off by 5 u; the bound is 8 u of the sum of magnitudes and the rounding to the type."""
    g = _gen(bag)
    table = (1.0 + torch.rand(vocab, dim, generator=g)).to(dtype)
    tok = torch.randint(0, vocab, (n, bag), generator=g)
    tok[:, 5] = -1
    scale = 2.0 ** -17  # (in fp16 the sums themselves are beyond the type)
    want = torch.stack([(table.double()[tok[i].clamp(min=0)] * (tok[i] >= 0)[:, None]).sum(0) * scale for i in range(n)])
    r = ROUND[dtype] + 8 * U
    for t in (tok, tok.int()):
        got = ctx.embed_tokens(table.cuda(), t.cuda(), scale).cpu().double()
        assert bool(((got - want).abs() <= r * want).all()), float(((got - want).abs() / want).max() / U)


def test_lookup_of_bags_with_infinite_rows(ctx):  # noqa: F811
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        table = torch.ones(4, 9).to(dtype)
        table[1], table[2], table[3] = float("inf"), float("-inf"), float("nan")
        tok = torch.zeros(4, 50, dtype=torch.int32)
        tok[0, 3], tok[1, 30], tok[2, 4], tok[2, 40], tok[3, 20] = 1, 2, 1, 2, 3
        got = ctx.embed_tokens(table.cuda(), tok.cuda()).cpu().float()
        assert bool((got[0] == math.inf).all()) and bool((got[1] == -math.inf).all()) and bool(torch.isnan(got[2:]).all())


@pytest.mark.parametrize("n,dim,vocab", [(2_000_003, 1024, 2), (4_000_003, 5, 1), (700_001, 264, 3)])
def test_lookup_gradient_of_very_frequent_tokens(ctx, n, dim, vocab):  # noqa: F811
    """Hundreds of thousands of rows of few distinct values per token, of one sign: units of 64 as trees of eight (11 u), four units at a time and a sum of these that keeps
    its roundings (5 u)."""
    g = torch.Generator(device="cuda").manual_seed(n)
    tok = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    kinds = (1.0 + torch.rand(7, dim, generator=g, device="cuda")).bfloat16()
    pick = torch.randint(0, 7, (n,), generator=g, device="cuda")
    grad = kinds[pick]
    got = ctx.embed_gradient(tok, grad, vocab, 2.0 ** -20)
    counts = torch.zeros(vocab, 7, dtype=torch.float64, device="cuda")
    counts.view(-1).scatter_add_(0, tok.long() * 7 + pick, torch.ones(n, dtype=torch.float64, device="cuda"))
    want = counts @ kinds.double() * 2.0 ** -20
    assert bool(((got.double() - want).abs() <= (2.0 ** -8 + 16 * U) * want).all())
    full = ctx.embed_gradient(tok[:400_000], grad[:400_000].float(), vocab, 2.0 ** -20)
    counts = torch.zeros(vocab, 7, dtype=torch.float64, device="cuda")
    counts.view(-1).scatter_add_(0, tok[:400_000].long() * 7 + pick[:400_000], torch.ones(400_000, dtype=torch.float64, device="cuda"))
    want = counts @ kinds.double() * 2.0 ** -20
    assert bool(((full.double() - want).abs() <= 17 * U * want).all()), float(((full.double() - want).abs() / want).max() / U)


# ---- where blocks and results lie ------------------------------------------------------------------------


def test_blocks_of_another_device_are_refused():
    """The context's number is changed instead of the tensors' device: a second card is not needed."""
    from paper_2207_09682_amd import Context
    c = Context(1, 1, 2, max_leaves=1, workspace_flags=0, device="cuda")
    assert c.device == torch.device("cuda", torch.cuda.current_device())
    scratch, norm = torch.empty(1 << 16, dtype=torch.uint8, device=c.device), torch.zeros(1, device=c.device)
    with pytest.raises(ValueError):
        c.clip_gradients([], 1.0, norm=torch.zeros(0, device=c.device))
    assert float(c.clip_gradients([], 1.0, norm=norm, scratch=scratch)) == 0.0
    stream = c._sync_stream
    c._index, c._sync_stream = c._index + 1, lambda: None
    try:
        with pytest.raises(ValueError):
            c.clip_gradients([], 1.0, scratch=scratch)
        with pytest.raises(ValueError):
            c.clip_gradients([], 1.0, norm=norm)
    finally:
        c._index, c._sync_stream = c._index - 1, stream


# ---- every kernel family: rows that hold anything, streams, graphs ----------------------------------------

# few rows; few rows against few classes; swept; weights where they lie, in tiles of 32, 64 and 128 rows; both second products at once; tiles, an odd number of rows; blocks of rows
FAMILIES = [(torch.bfloat16, 9, 264, 3000), (torch.bfloat16, 16, 2048, 26_000), (torch.bfloat16, 200, 250, 700), (torch.bfloat16, 33, 300, 200), (torch.bfloat16, 301, 520, 1000),
            (torch.bfloat16, 2101, 264, 2300), (torch.float32, 3, 40, 500), (torch.float32, 15, 770, 12_500), (torch.float32, 200, 100, 700), (torch.float32, 20, 192, 3000),
            (torch.float32, 64, 260, 9000), (torch.float32, 120, 1000, 12_000), (torch.float32, 701, 300, 1200), (torch.float32, 2101, 264, 2300)]


@pytest.mark.parametrize("dtype,n,dim,vocab", FAMILIES)
def test_left_out_rows_may_hold_anything_in_every_family(ctx, dtype, n, dim, vocab):  # noqa: F811
    """Rows without target hold NaN, rows of weight 0 infinities: the other rows' results and the class weights' gradient are the same bits; a live row of NaN poisons its own
    row and the class weights' gradient, and no other row."""
    x, w, t, u = _problem(n, dim, vocab, dtype)
    t[0], t[1], u[2], t[2], u[n - 1], t[n - 1] = 1, -1, 0.0, 3, 1.0, 2  # (the last row counts: rows behind it are read as it)
    u[0] = 0.5
    ok = (t >= 0) & (t < vocab)
    live = ok & (u != 0)
    loss, lse = ctx.softmax_loss(x.cuda(), w.cuda(), t.cuda())
    want = ctx.softmax_gradients(x.cuda(), w.cuda(), t.cuda(), lse, u.cuda())
    bad = x.clone()
    bad[~ok], bad[ok & (u == 0)] = float("nan"), float("inf")
    loss2, lse2 = ctx.softmax_loss(bad.cuda(), w.cuda(), t.cuda())
    assert torch.equal(lse2.cpu()[live], lse.cpu()[live]) and torch.equal(loss2.cpu()[live], loss.cpu()[live]) and bool((loss2.cpu()[~ok] == 0).all())
    got = ctx.softmax_gradients(bad.cuda(), w.cuda(), t.cuda(), lse2, u.cuda())
    assert torch.equal(got[0].cpu()[live], want[0].cpu()[live]) and bool((got[0].cpu()[~live] == 0).all()) and torch.equal(got[1], want[1])
    for row in (0, n - 1):
        bad = x.clone()
        bad[row] = float("nan")
        keep = torch.arange(n) != row
        loss2, lse2 = ctx.softmax_loss(bad.cuda(), w.cuda(), t.cuda())
        assert bool(torch.isnan(lse2[row])) and torch.equal(lse2.cpu()[keep], lse.cpu()[keep]) and torch.equal(loss2.cpu()[keep], loss.cpu()[keep])
        got = ctx.softmax_gradients(bad.cuda(), w.cuda(), t.cuda(), lse2, u.cuda())
        assert bool(torch.isnan(got[0][row]).all()) and torch.equal(got[0].cpu()[keep], want[0].cpu()[keep]) and bool(torch.isnan(got[1]).all())


@pytest.mark.parametrize("dtype,n,dim,vocab", FAMILIES)
def test_rows_that_lie_apart_in_every_family(ctx, dtype, n, dim, vocab):  # noqa: F811
    x, w, t, u = _problem(n, dim, vocab, dtype)
    xs, ws = torch.full((n, dim + 11), float("nan"), dtype=dtype), torch.full((vocab, dim + 5), float("nan"), dtype=dtype)
    xs[:, :dim], ws[:, :dim] = x, w
    args, apart = (x.cuda(), w.cuda(), t.cuda()), (xs.cuda()[:, :dim], ws.cuda()[:, :dim], t.cuda())
    want, got = ctx.softmax_loss(*args), ctx.softmax_loss(*apart)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    a, b = ctx.softmax_gradients(*args, want[1], u.cuda()), ctx.softmax_gradients(*apart, want[1], u.cuda())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype,n,dim,vocab", FAMILIES)
def test_graphs_and_streams_in_every_family(ctx, dtype, n, dim, vocab):  # noqa: F811
    x, w, t, u = (a.cuda() for a in _problem(n, dim, vocab, dtype))
    e = lambda *s, d=dtype: torch.zeros(s, dtype=d, device="cuda")  # noqa: E731
    room = lambda: (e(n, d=torch.float32), e(n, d=torch.float32), e(n, dim), e(vocab, dim))  # noqa: E731

    def step(o):
        loss, lse = ctx.softmax_loss(x, w, t, loss=o[0], lse=o[1])
        ctx.softmax_gradients(x, w, t, lse, u, grad_x=o[2], grad_weight=o[3])

    want, other, rec = room(), room(), room()
    step(want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step(other)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(other, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(rec)
    for k in range(3):
        if k:
            x.copy_(x * 0.5 + 0.25)
        if k == 2 and dtype == torch.float32:
            x[:, 0] *= 1e9  # (fp32: the range of the rows decides in the kernels, not when they are recorded)
            w[:, 0] *= 1e-9
        step(want)
        for r in rec:
            r.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(rec, want)), k
