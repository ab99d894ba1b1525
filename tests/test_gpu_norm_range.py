"""8-bit rows of the norm whose products h w lie past an end of binary32, though h rstd w does not: scales and codes against 64 bits.

Tolerances as in test_gpu_norm.py: rstd off by (H / 64 + 16) 2^-25 at most, four roundings to y and eight more to a code and back."""
import pytest
import torch

import layers_ref as ref
from paper_2104_08378_amd import sp24

pytestmark = pytest.mark.gpu

BF16, F32, I8, F8 = torch.bfloat16, torch.float32, torch.int8, torch.float8_e4m3fn


# sizes of rows and weights: products of 2^126 to 2^152 and of 2^-153 to 2^-120, and some between; the squares and their sum stay within binary32
@pytest.mark.parametrize("rows,weights", [(2.0 ** 50, 2.0 ** 84), (2.0 ** 54, 2.0 ** 98), (2.0 ** 54, 2.0 ** 72), (2.0 ** 20, 2.0 ** -20),
                                          (2.0 ** -50, 2.0 ** -70), (2.0 ** -55, 2.0 ** -90), (2.0 ** -58, 2.0 ** -95)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("out", [I8, F8])
@pytest.mark.parametrize("N,H", [(3, 77), (2, 512), (1030, 1024), (1, 8192), (2, 20000)])
def test_products_past_the_ends_of_binary32(N, H, out, dtype, rows, weights):
    g = torch.Generator().manual_seed(N + H)
    x = (torch.randn(N, H, generator=g) * rows).to(dtype).cuda()
    w = (0.5 + torch.rand(H, generator=g)).mul(weights).cuda()
    n = sp24.sp24_rmsnorm(x, w, 0.0, out_dtype=out)
    want, err = ref.norm(x, w, 0.0)[2], (H / 64 + 16) * 2.0 ** -25 + 4 * 2.0 ** -24 + 2.0 ** -21
    top = want.abs().amax(1).clamp(min=2.0 ** -100)
    ref.close(n.scale, top / ref.TOP[out], err * top / ref.TOP[out], "scale")
    codes, exact = ref.d(n.y), want / (top / ref.TOP[out])[:, None]
    # half a code; half a unit of three fraction bits, or half the smallest step
    room = torch.tensor(0.5) if out == I8 else torch.maximum(exact.abs() * 2.0 ** -4, torch.tensor(2.0 ** -10))
    assert bool(((codes - exact).abs() <= room * (1 + 1e-5) + 2 * err * ref.TOP[out]).all())
