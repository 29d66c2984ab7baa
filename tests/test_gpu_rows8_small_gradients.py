"""Weight gradients of half-precision numbers below its least normal one, 2^-14, and of rows whose scales put them there: with scales that are powers
of two nothing of a product is lost, whatever its size."""
import zlib

import pytest
import torch

import operators_util as R
import paper_2111_00705_amd as P
import rows8_util as Q

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def small_rows(g, rows, cols, outs, power):
    """(dy with a standard deviation of 2^power and every seventh channel common, q, scales of 2^-21 to 2^1)"""
    dy = torch.randn(rows, outs, generator=g) * 2.0 ** power
    dy[:, ::7] = torch.randn(rows, len(range(0, outs, 7)), generator=g) * 0.1
    q = torch.randint(-127, 128, (rows, cols), generator=g).to(torch.int8)
    return dy.to(F16), q, torch.ldexp(torch.ones(rows), torch.randint(-21, 2, (rows,), generator=g))


@pytest.mark.parametrize("power", [-24, -20, -14])
@pytest.mark.parametrize("n,cols,outs", [(5, 40, 48), (3, 130, 257), (2, 700, 9)])
def test_a_product_is_exact(n, cols, outs, power):
    """Workers of one row.  A product of 11 and 7 bits has 18: so have its parts and their sum, which fp32 holds."""
    print(f"[case] one row {n} {cols}->{outs} 2^{power}", flush=True)
    dy, q, scale = small_rows(gen("one", n, cols, outs, power), n, cols, outs, power)
    want = dy.double()[:, :, None] * (q.double() * scale.double()[:, None])[:, None, :]
    for turned in (False, True):
        dw = torch.zeros(n, cols, outs, device="cuda").transpose(1, 2) if turned else torch.zeros(n, outs, cols, device="cuda")
        P.linear_weight_grad(dy.cuda(), q.cuda(), scale.cuda(), dw, binary=True)
        assert torch.equal(dw.cpu().double(), want)


@pytest.mark.parametrize("power", [-24, -20, -14])
@pytest.mark.parametrize("n,per,cols,outs", [(2, 33, 16, 130), (2, 300, 129, 127), (1, 4200, 64, 72), (1, 96, 1300, 700)])
def test_sums_are_off_by_their_additions_only(n, per, cols, outs, power):
    """(per + 64) roundings of 2^-24 of the sum of the products' sizes: the bound of numbers of common sizes."""
    print(f"[case] sums {n}x{per} {cols}->{outs} 2^{power}", flush=True)
    dy, q, scale = small_rows(gen("sums", n, per, cols, outs, power), n * per, cols, outs, power)
    dw, db, s_dw, s_db = Q.weight_grad(dy, q, scale, n, True)
    for grad in (F32, BF16):
        place = torch.full((n, outs * cols + outs), 7.0, dtype=grad, device="cuda")
        w, b = place[:, :outs * cols].unflatten(1, (outs, cols)), place[:, outs * cols:]
        P.linear_weight_grad(dy.cuda(), q.cuda(), scale.cuda(), w, b, binary=True)
        R.close(w, dw, s_dw, f"dweight {grad}")
        R.close(b, db, s_db, "dbias")
