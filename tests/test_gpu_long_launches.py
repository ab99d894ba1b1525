"""Row counts (and one number of features) at which a workgroup to every piece of work would be a launch of 2^32 threads and more, which runs a
fraction of them and reports nothing: small values whose sums are exact, compared bit for bit on the GPU."""
import pytest
import torch

from paper_2104_08378_amd import sp24

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
ROWS = (1 << 26) + 5                                  # of one value: 64 threads a row


@pytest.fixture(autouse=True)
def release():
    yield
    torch.cuda.empty_cache()


def whole(shape, lo, hi, dtype):
    g = torch.Generator(device="cuda").manual_seed(sum(shape))
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32 if dtype == torch.int32 else torch.int8).to(dtype)


def test_gather():
    x, scale, rows = whole((1000, 1), -100, 100, BF16), whole((1000,), 1, 100, F32), whole((ROWS,), -1, 999, torch.int32)
    xs, scales = sp24.sp24_moe_gather(x, rows, 1, scale=scale)
    live = rows >= 0
    at = rows.clamp(min=0).long()
    assert torch.equal(xs[:, 0], torch.where(live, x[at, 0], 0)) and torch.equal(scales, torch.where(live, scale[at], 0))


def test_combine():
    y, slots, weights = whole((1000, 1), -100, 100, BF16), whole((ROWS, 1), -1, 1000, torch.int32), whole((ROWS, 1), -2, 2, F32)
    out = sp24.sp24_moe_combine(y, slots, weights)
    live = (slots >= 0) & (slots < 1000)
    assert torch.equal(out, torch.where(live, y[slots.clamp(0, 999).long(), 0].float() * weights, 0).to(BF16))


def test_combine_gradients():
    N = 1000
    dout, y, weights = whole((N, 1), -100, 100, BF16), whole((ROWS, 1), -100, 100, BF16), whole((N, 1), -2, 2, F32)
    rows = torch.full((ROWS,), -1, dtype=torch.int32, device="cuda")
    at = (torch.arange(N, device="cuda") * (ROWS // N + 1)).clamp(max=ROWS - 1)          # the last ones in the last row
    at[-1], at[-2] = ROWS - 1, ROWS - 2
    rows[at] = torch.arange(N, device="cuda", dtype=torch.int32)
    slots = torch.full((N, 1), -1, dtype=torch.int32, device="cuda")
    slots[rows[at].long(), 0] = at.to(torch.int32)
    dy, dw = sp24.sp24_moe_combine_backward(dout, y, slots, rows, weights)
    live = rows >= 0
    choice = rows.clamp(min=0).long()
    assert torch.equal(dy[:, 0], torch.where(live, dout[choice, 0].float() * weights[choice, 0], 0).to(BF16))
    named = torch.zeros(N, dtype=torch.bool, device="cuda")
    named[rows[live].long()] = True
    assert bool(named.all())
    assert torch.equal(dw, dout.float() * y[slots[:, 0].long()].float())


@pytest.mark.parametrize("act,N", [("none", (1 << 30) + 3), ("relu", (1 << 29) + 7)])
def test_gradient_of_a_layers_result_on_many_rows(act, N):
    """Tiles of 64 rows, 256 and 512 threads.  (z is dy: what ReLU leaves adds up to 2^27, in 32 sums that are exact and 31 roundings.)"""
    dy = whole((N, 1), -1, 1, BF16)
    z = None if act == "none" else whole((N, 1), -1, 1, BF16)
    dz, dzt, db = sp24.sp24_linear_backward(dy, z, act)
    want = dy if z is None else torch.where(z > 0, dy, 0)
    assert torch.equal(dz, want) and torch.equal(dzt[0], want[:, 0])
    total = sum(int(part.to(torch.int32).sum()) for part in want[:, 0].split(1 << 26))
    assert abs(float(db[0]) - total) <= (0 if act == "none" else 31 * 2.0 ** -24 * total) and abs(total) < (1 << 24 if act == "none" else 1 << 28)


def test_bias_gradient_of_many_features():
    M = (1 << 27) + 5
    dy = whole((2, M), -100, 100, BF16)
    dz, dzt, db = sp24.sp24_linear_backward(dy, None, "none")
    assert torch.equal(db, dy[0].float() + dy[1].float()) and torch.equal(dzt[:, 1], dy[1])
