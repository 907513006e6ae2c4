"""MX operators at the ends of their ranges."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import mx_oracle as mx  # noqa: E402
from paper_2511_04063_amd import binding as B  # noqa: E402
from test_gpu_mx import TYPES, rng, up  # noqa: E402


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    c.ensure_workspace(1, 256, 512, B.DQ_F32)
    yield c
    torch.cuda.synchronize()
    c.close()


# ----------------------------------------------------------------------------------- objective
@pytest.mark.parametrize("grad", [B.DQ_F32, B.DQ_BF16])
@pytest.mark.parametrize("obj,fmt", [(B.DQ_OBJ_MXFP4, mx.MXFP4), (B.DQ_OBJ_MXFP8, mx.MXFP8)])
@pytest.mark.parametrize("where", ["large", "small"])
def test_objective_whose_squares_leave_fp32(ctx, obj, fmt, grad, where):
    """Errors whose squares, or sums of four of them, lie beyond fp32's largest or below its smallest normal number, and a loss that does not.
    The bounds are those of ordinary rows: the sums are formed in 64 bits, so only the roundings of the loss and of the gradient count."""
    g = rng(77)
    if where == "large":
        T, n, mode = 6, 4096, "mean"
        Y = g.standard_normal((T, n)).astype(np.float32)
        # one block a row: with e4m3 errors reach 2^-4 of the values, with e2m1 a quarter
        Y[:, 64:96] *= np.float32(2.0 ** 68 if fmt == mx.MXFP8 else 2.0 ** 66)
        Y[0, 64:68] = np.float32(1.06 * 2.0 ** 71 if fmt == mx.MXFP8 else 1.24 * 2.0 ** 68)
    else:
        T, n, mode = 3000, 96, "sum"
        Y = (g.standard_normal((T, n)) * 2.0 ** (-63 if fmt == mx.MXFP8 else -64)).astype(np.float32)
    ref_loss, ref = mx.objective(Y, fmt, mode)
    e2 = (ref / (2.0 / n * (1.0 / T if mode == "mean" else 1.0))) ** 2
    largest = np.finfo(np.float32).max
    assert (e2.reshape(T, -1, 4).sum(-1).max() > largest if where == "large" else e2.max() < 2.0 ** -126) and 2.0 ** -126 < ref_loss < largest
    buf = torch.empty((T, up(n, 8)), dtype=TYPES[grad], device="cuda")[:, :n]
    loss = torch.zeros(1, device="cuda")
    red = B.DQ_REDUCE_TOKEN_MEAN if mode == "mean" else B.DQ_REDUCE_SUM
    ctx.dq_objective_loss_grad(obj, 4, torch.from_numpy(Y).cuda(), red, loss, buf, grad)
    assert abs(loss.item() - ref_loss) <= 8 * 2.0 ** -24 * ref_loss
    assert (np.abs(buf.double().cpu().numpy() - ref) <= np.abs(ref) * (4 * 2.0 ** -24 + (2.0 ** -8 if grad == B.DQ_BF16 else 0.0))).all()
    assert ctx.dq_device_flags() == 0
