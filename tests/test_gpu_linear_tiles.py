"""The linear layers' larger tiles and their splits at sizes that no tile divides, in every
form of the epilogue, against the definition in 64 bits.

By the cost that chooses them, of the products below (tokens, rows, cols):
  1556 x 17821 x 7456 and 7459   256 x 256 whole in every direction, ends in all three
                                 sizes; of 7459 with padded copies
  4675 x 439 x 19008             forward 256 x 256 in 4 splits
  1102 x 1432 x 3488             forward 256 x 128 in 4 splits, dx and dweight 256 x 128
  1000 x 520 x 9001              forward 256 x 128 in 9 splits, of padded copies
  2428 x 11184 x 64              dx 256 x 256 in 25 splits, dweight in 5
  7345 x 840 x 1440              dweight 256 x 128 in 6 splits, dx 256 x 256
  2005 x 22192 x 183             dx 256 x 256 in 22 splits, dweight 256 x 256 in 2 or 256 x 128
  520 x 4000 x 4100              forward 256 x 256 in 4 splits, dx 256 x 128 in 3
  333 x 8200 x 520               dx 256 x 128 in 22 or 26 splits, the last one shorter
  2000 x 2056 x 1501             dx and dweight 256 x 128, in 2 splits for d of two parts
The tolerances are test_gpu_linear.py's and test_gpu_linear_gradient.py's.
"""
import pytest
import torch

from paper_2602_03839_amd import head

from test_gpu_linear import ACTS, forward64, gen, make, normal, within
from test_gpu_linear_gradient import check

pytestmark = pytest.mark.gpu

SIZES = [(1556, 17821, 7456), (1556, 17821, 7459), (4675, 439, 19008), (1102, 1432, 3488), (1000, 520, 9001),
         (2428, 11184, 64), (7345, 840, 1440), (2005, 22192, 183), (520, 4000, 4100), (333, 8200, 520), (2000, 2056, 1501)]


@pytest.mark.parametrize("typ", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,rows,cols", SIZES)
def test_forward(tokens, rows, cols, typ):
    """An activation after the other, so that each meets both types and most tiles; with
    everything, in place of the residual and of the multiplier, and with nothing."""
    for k in range(3):
        act = ACTS[(SIZES.index((tokens, rows, cols)) + 2 * k + (typ is torch.float32)) % 5]
        x, w, b, t, r, _ = make(tokens, rows, cols, typ, rows + k, bias=k != 2, times=k != 2, residual=k != 2,
                                bias_type=torch.bfloat16 if k == 1 else torch.float32)
        h = head.Linear(w, b, activation=act, max_tokens=tokens)
        y, pre = h(x, residual=r, times=t, keep_pre=True, out_dtype=typ)
        ey, yerr, epre, perr = forward64(x, w, b, act, t, r, typ)
        within(y, ey, yerr, "y")
        within(pre, epre, perr, "pre")
        del ey, yerr, epre, perr, pre
        if k == 0:
            out = r.clone()
            assert torch.equal(h(x, residual=out, times=t, out=out), y) and torch.equal(out, y)
        elif k == 1:
            out = t.clone()
            assert torch.equal(h(x, residual=r, times=out, out=out), y) and torch.equal(out, y)


@pytest.mark.parametrize("tokens,rows,cols", SIZES)
def test_backward(tokens, rows, cols):
    """d of two parts from FP32 and BF16 gradients, and of one."""
    first = SIZES.index((tokens, rows, cols))
    for k, (typ, with_times) in enumerate(((torch.float32, False), (torch.bfloat16, True), (torch.bfloat16, False))):
        act = None if k == 2 else ACTS[(first + k) % 5]
        x, w, b, t, _, dy = make(tokens, rows, cols, typ, rows + k, times=with_times, residual=False)
        pre = normal(gen(k), tokens, rows).to(typ) if act or with_times else None
        h = head.Linear(w, b, activation=act, max_tokens=tokens)
        check(h, x, w, dy, pre, t, act, exact=k == 2)


@pytest.mark.parametrize("tokens,rows,cols", [(1556, 2821, 1000), (4675, 439, 19008), (1102, 1432, 3488)])
def test_strided_rows(tokens, rows, cols):
    """Rows that lie apart, at 16 bytes and not, leave what is between them as it was."""
    for typ in (torch.bfloat16, torch.float32):
        for apart in (24, 5):
            x, w, b, t, r, dy = make(tokens, rows, cols, typ, 6)
            h = head.Linear(w, b, activation="silu", max_tokens=tokens)

            def view(like):
                buf = torch.full((tokens, like.shape[1] + apart), 7.0, dtype=like.dtype, device="cuda")
                buf[:, :like.shape[1]] = like
                return buf[:, :like.shape[1]], buf

            (xv, _), (tv, _), (rv, _), (dv, _) = map(view, (x, t, r, dy))
            (yv, yb), (pv, pb), (dtv, dtb) = (view(torch.zeros_like(dy)) for _ in range(3))
            dxv, dxb = view(torch.zeros_like(x))
            want, want_pre = h(x, residual=r, times=t, keep_pre=True, out_dtype=typ)
            h(xv, residual=rv, times=tv, out=yv, pre=pv)
            tol = 2.0 ** -7 if typ is torch.bfloat16 else 1e-5
            within(yv, want.double(), tol * (1 + want.double().abs()), "y")
            within(pv, want_pre.double(), tol * (1 + want_pre.double().abs()), "pre")
            want = h.backward(dy, x, pre=want_pre, times=t)
            got = h.backward(dv, xv, pre=want_pre, times=tv, dx=dxv, dtimes=dtv)
            for a, e in zip(got, want):
                within(a, e.double(), 2.0 ** -7 * (e.double().abs() + e.double().abs().mean()), "gradient")
            for buf, n in ((yb, rows), (pb, rows), (dtb, rows), (dxb, cols)):
                assert (buf[:, n:] == 7).all()
