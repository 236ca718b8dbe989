"""Layers of experts near the end of fp32's range, which is bf16's."""
import pytest

torch = pytest.importorskip("torch")

from paper_2503_00784_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FORMS = pytest.mark.parametrize("scaled", [False, True])
D, FF = 128, 96


def _layer(gate, up, down, n, top_k, scaled):
    """n equal experts: rows that are x[0] times the first unit vector have hidden values silu(x0 * gate) * (x0 * up) in channel 5 and zeros in the others,
    and outputs that are down times that, with the sign of the output's number."""
    g, u, w = torch.zeros((FF, D)), torch.zeros((FF, D)), torch.zeros((D, FF))
    g[5, 0], u[5, 0] = gate, up
    w[:, 5] = down * torch.where(torch.arange(D) % 2 == 0, 1.0, -1.0)
    expert = tuple(m.to(torch.bfloat16).to(DEV) for m in (g, u, w))
    return B.ExpertLayer(torch.zeros((n, D), dtype=torch.bfloat16, device=DEV), [expert] * n, top_k, scaled=scaled)


def _rows(rows, first):
    x = torch.zeros((rows, D))
    x[:, 0] = first
    return x.to(torch.bfloat16).to(DEV)


@FORMS
@pytest.mark.parametrize("n,rows", [(1, 3), (4, 5), (1, 20), (1, 40)])
def test_hidden_values_between_the_largest_of_bf16_and_of_fp32(n, rows, scaled):
    """(181 / 128)^2 * 2^127 is below fp32's largest number and rounds to 2^128 in bf16.  The pair keeps 2^-16 of a hidden value, and the output, of the
    size of 2^28, is rounded to bf16."""
    x0 = 181.0 / 128.0
    layer = _layer(2.0 ** 64, 2.0 ** 63, 2.0 ** -100, n, 1, scaled)
    y = layer.run(_rows(rows, x0))[0].cpu().double()
    want = x0 * 2.0 ** 64 * x0 * 2.0 ** 63 * 2.0 ** -100 * torch.where(torch.arange(D) % 2 == 0, 1.0, -1.0).double()
    assert bool(((y - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -15)).all()), y[0, :4]


@FORMS
@pytest.mark.parametrize("n,top_k,rows", [(1, 1, 3), (1, 1, 20), (1, 1, 40), (4, 2, 5)])
def test_hidden_values_beyond_fp32_are_infinite(n, top_k, rows, scaled):
    """2^140 is an infinity in fp32, and so is what it is multiplied with, up to the sign; rows beside it stay as they are."""
    layer = _layer(2.0 ** 70, 2.0 ** 70, 2.0 ** -50, n, top_k, scaled)
    x = _rows(rows, 1.0)
    x[1, 0] = 2.0 ** -60  # silu(2^10) * 2^10
    y = layer.run(x)[0].cpu().double()
    sign = torch.where(torch.arange(D) % 2 == 0, 1.0, -1.0).double()
    keep = [r for r in range(rows) if r != 1]
    assert torch.equal(y[keep], (sign * torch.inf).expand(len(keep), D))
    assert torch.equal(y[1], sign * 2.0 ** -30)


@pytest.mark.parametrize("n,rows", [(1, 3), (1, 20), (1, 40)])
@FORMS
def test_rows_near_the_largest(n, rows, scaled):
    """Rows of 1.5 * 2^126 under gates and ups that bring them to 1.5 * 2^26 and 1.5 * 2^24: products with what the matrices stand for, far from the end of
    fp32, whatever scale the 8-bit blocks have (2^-100 is 256 * 2^-108 there)."""
    layer = _layer(2.0 ** -100, 2.0 ** -102, 2.0 ** -50, n, 1, scaled)
    y = layer.run(_rows(rows, 1.5 * 2.0 ** 126))[0].cpu().double()
    want = 2.25 * torch.where(torch.arange(D) % 2 == 0, 1.0, -1.0).double()
    assert torch.equal(y, want.expand(rows, D))
