"""Fp8Linear (paper_2503_06564_amd/fp8_block.py) at fewer rows than it was made for: a smaller last batch, one token, none.  Every product is
the same call as of a linear made for that many rows, so the bits are the same."""
import pytest
import torch

from paper_2503_06564_amd import fp8_block, trdq

pytestmark = pytest.mark.gpu


def run(lin, x, dy):
    rows, (out, inn) = x.shape[0], lin.W.shape
    y, dx = (torch.full((rows, n), 9.0, dtype=torch.bfloat16, device="cuda") for n in (out, inn))
    codes = fp8_block._codes(rows, inn, "e4m3", "cuda")
    trdq.fp8_quant(x, *codes)
    lin.forward(*codes, y)
    lin.backward(x, dy, dx)
    torch.cuda.synchronize()
    return y, dx, lin.dW.clone(), lin.db.clone()


@pytest.mark.parametrize("out,inn,tokens", [(1152, 4608, 4096), (771, 200, 300)])
def test_fewer_rows_than_tokens(out, inn, tokens):
    g = torch.Generator().manual_seed(5)
    W, b = (torch.randn(out, inn, generator=g) * inn ** -0.5).to("cuda"), torch.randn(out, generator=g).to("cuda")
    lin = fp8_block.Fp8Linear(W, b, tokens)
    for rows in (tokens, 276, 129, 33, 1, 0, tokens - 1):
        x, dy = (torch.randn(rows, n, generator=g).to("cuda").to(torch.bfloat16) for n in (inn, out))
        got = run(lin, x, dy)
        if rows == 0:
            assert bool((got[2] == 0).all()) and bool((got[3] == 0).all())
            continue
        want = run(fp8_block.Fp8Linear(W, b, rows), x, dy)
        for name, a, c in zip(("y", "dx", "dW"), got, want):
            assert torch.equal(a.view(torch.uint8), c.view(torch.uint8)), (rows, name)
        # db: the same sums by a library product
        want = dy.double().sum(0)
        assert bool(((got[3].double() - want).abs() <= (rows + 8) * 2.0 ** -24 * dy.double().abs().sum(0)).all()), rows
