"""fp32 values as sums of smaller ones, on the CPU: inputs that show any product of pieces which is left out, and the bound that tells whether rows may be held in two fp16 pieces."""
import pytest
import torch

U = 2.0 ** -24
SIX = [(2, 0), (1, 1), (0, 2), (1, 0), (0, 1), (0, 0)]  # three bfloat16 pieces
THREE = [(1, 0), (0, 1), (0, 0)]                        # two fp16 ones


def coherent(rows, dim, seed):
    """Positive values whose three bfloat16 pieces are all positive and as large as they may be for all of them alike (2^e times 1 + k / 128, 1.5 2^-10 and 1.5 2^-19), so that what
    is left out of their products adds up and nothing averages out."""
    g = torch.Generator().manual_seed(seed)
    k = torch.randint(0, 32, (rows, dim), generator=g).double()
    return (0.25 * (1.0 + k / 128.0 + 1.5 * 2.0 ** -10 + 1.5 * 2.0 ** -19)).float()


def _pieces(v, dtype, count):
    out, rest = [], v.double()
    for _ in range(count):
        out.append(rest.to(dtype).double())
        rest = rest - out[-1]
    return out


def _halves(v):
    """Two fp16 pieces of each row, brought to 2^14 .. 2^15 by a power of two and back."""
    by = 2.0 ** (14 - torch.floor(torch.log2(v.double().abs().amax(1, keepdim=True))))
    return [p / by for p in _pieces((v.double() * by).float(), torch.float16, 2)]


@pytest.mark.parametrize("dim", [64, 192, 264])
def test_any_product_that_is_left_out_shows(dim):
    """More than 16 u of the sum of magnitudes and 16 u: what test_no_piece_of_fp32_values_is_lost allows."""
    x, w = coherent(30, dim, 1), coherent(40, dim, 2)
    exact = x.double() @ w.double().t()
    for x_pieces, w_pieces, products in ((_pieces(x, torch.bfloat16, 3), _pieces(w, torch.bfloat16, 3), SIX), (_halves(x), _halves(w), THREE)):
        whole = sum(x_pieces[a] @ w_pieces[b].t() for a, b in products)
        assert bool(((whole - exact).abs() <= 4 * U * exact).all())
        for a, b in products:
            missing = whole - x_pieces[a] @ w_pieces[b].t()
            assert bool(((missing - exact).abs() > 16 * U * (exact + 1)).all()), (a, b)


def _marks(v):
    """loose, faint: as the layout of the kernels has them."""
    b = v.abs()
    top = b.amax(1, keepdim=True)
    alive = top > 0
    loose = alive[:, 0] & (4 * (b < top * 2.0 ** -9).sum(1) > v.shape[1])
    faint = alive & (b > 0) & (b < top * 2.0 ** -17)
    return bool(loose.any()), bool(faint.any())


@pytest.mark.parametrize("dim", [1, 4, 7, 40, 264])
def test_bound_of_two_fp16_pieces(dim):
    """Rows that the rule leaves in two pieces: within 20 u of the sum of magnitudes, with values spread over many orders of magnitude, at the limits of the rule and against rows
    chosen to meet their faint values."""
    g = torch.Generator().manual_seed(dim)
    taken = 0
    for trial in range(300):
        small = torch.rand(2, 30, dim, generator=g) < 0.25 * torch.rand(1, generator=g)
        spread = torch.where(small, 2.0 ** -(9 + 40 * torch.rand(2, 30, dim, generator=g)), 2.0 ** -(9 * torch.rand(2, 30, dim, generator=g) * torch.rand(1, generator=g)))
        v = ((1.0 + torch.rand(2, 30, dim, generator=g)) * spread * torch.sign(torch.randn(2, 30, dim, generator=g))).float()
        x, w = v[0], v[1]
        if trial % 3 == 0:
            w = torch.where(x.abs() < x.abs().amax(1, keepdim=True) * 2.0 ** -9, w.abs().amax(1, keepdim=True), w * 2.0 ** -8)  # (large where x is small)
        (lx, fx), (lw, fw) = _marks(x), _marks(w)
        if (lx or lw) and (fx or fw):
            continue
        taken += 1
        exact, size = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()
        xs, ws = _halves(x), _halves(w)
        got = sum(xs[a] @ ws[b].t() for a, b in THREE)
        assert bool(((got - exact).abs() <= 20 * U * size).all())
    assert taken > 5
