"""The layers around the gradient exchange where numbers, sizes and callers go to their ends: scales near the ends of binary32, long sums of
weights' gradients, every shape of workgroup over several steps, second rows and second tiles, long launches of every type."""
import math

import pytest
import torch

import paper_2305_18627_amd as gq
import test_layer_operators as L

gpu = pytest.mark.gpu
DEV, U, TYPES, close = L.DEV, L.U, L.TYPES, L.close


def device_weights(g, rows, cols, group, st):
    """Random codes and scales made on the GPU: (codes as numbers, packed, scales)."""
    q = torch.zeros(rows, 2 * gq.w4_row_bytes(cols), dtype=torch.int16, device=DEV)
    q[:, :cols] = torch.randint(-8, 8, (rows, cols), generator=g, device=DEV, dtype=torch.int16)
    codes = ((q[:, 0::2] & 15) | ((q[:, 1::2] & 15) << 4)).to(torch.uint8)
    scales = (0.01 + torch.rand(rows, -(-cols // group), generator=g, device=DEV)).to(st)
    return q[:, :cols], codes, scales


def exact_matvec(x, xs, q, scales, group):
    """(y in 64 bits, its tolerance before the output's rounding), a group of columns at a time: the roundings that plain_matvec counts."""
    y, off = (torch.zeros(x.shape[0], q.shape[0], dtype=torch.float64, device=DEV) for _ in range(2))
    for k in range(scales.shape[1]):
        at, s = slice(k * group, min((k + 1) * group, q.shape[1])), scales[:, k].double()
        xg = x[:, at].double()
        part = (xg @ q[:, at].double().t().contiguous()) * s
        y += part
        off += (scales.shape[1] + 3) * U * part.abs()
        if xs is None:
            off += (group + 4) * U * 32 * xg.abs().sum(1, keepdim=True) * s.abs()
    return (y, off) if xs is None else (y * xs.double()[:, None], off * xs.double()[:, None].abs())


# ---- the product near the ends of binary32 --------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 3, 12, 40, 100])
def test_int8_product_under_subnormal_scales_of_rows(m, group):
    """Scales of rows that a norm of tiny rows writes: subnormal, so that a product with a power of two would round them."""
    g = torch.Generator(DEV).manual_seed(m)
    q, codes, scales = device_weights(g, 200, 300, group, torch.float32)
    scales *= 2.0 ** 30
    x = torch.randint(-127, 128, (m, 300), generator=g, device=DEV).to(torch.int8)
    xs = ((16 * torch.arange(1000, 1000 + m, dtype=torch.float64) + 8) * 2.0 ** -149).float().to(DEV)
    y = torch.empty(m, 200, device=DEV)
    gq.w4_matvec(x, codes, scales, group, y, x_scales=xs)
    close(y, *exact_matvec(x, xs, q, scales, group))


@gpu
@pytest.mark.parametrize("m", [1, 3, 12, 40, 100])
@pytest.mark.parametrize("cols", [32, 64])
def test_int8_product_of_sums_near_the_end_of_binary32(cols, m):
    """Scales of weights under which the sum is below 2^126, and scales of rows that bring it back."""
    codes = torch.full((70, gq.w4_row_bytes(cols)), 0x77, dtype=torch.uint8, device=DEV)
    scales = torch.full((70, 1), 2.0 ** 110, device=DEV)
    x = torch.full((m, cols), 127, dtype=torch.int8, device=DEV)
    xs = torch.full((m,), 2.0 ** -10, device=DEV)
    y = torch.empty(m, 70, device=DEV)
    gq.w4_matvec(x, codes, scales, 64, y, x_scales=xs)
    want = torch.full((m, 70), 7.0 * 127 * cols * 2.0 ** 100, dtype=torch.float64)
    close(y, want, 2 * U * want)


def test_row_bytes_of_more_columns_than_the_calls_take():
    assert gq.w4_row_bytes(1 << 24) == 1 << 23 and gq.w4_row_bytes((1 << 24) + 1) == 0 and gq.w4_row_bytes(1 << 40) == 0


@gpu
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 5, 12, 40, 100])
def test_products_of_large_finite_rows_are_numbers(m, group):
    """bfloat16 rows whose sums of 24 |x| are beyond binary32, though their products are not; rows beside them keep their bits."""
    g = torch.Generator(DEV).manual_seed(m + group)
    rows, cols = 150, 300
    q, codes, scales = device_weights(g, rows, cols, group, torch.float32)
    scales *= 2.0 ** -20
    x = torch.randn(m, cols, generator=g, device=DEV).to(torch.bfloat16)
    clean = torch.empty(m, rows, device=DEV)
    gq.w4_matvec(x, codes, scales, group, clean)
    large = torch.arange(m, device=DEV) % 3 == 0
    x[large] = (x[large].float() * 2.0 ** 125).to(torch.bfloat16)
    assert torch.isfinite(x).all()
    y = torch.empty(m, rows, device=DEV)
    gq.w4_matvec(x, codes, scales, group, y)
    want, tol = exact_matvec(x, None, q, scales, group)
    assert float(want.abs().max()) < 2.0 ** 126
    close(y, want, tol)
    assert torch.equal(y[~large], clean[~large])
    # where the product itself is beyond binary32 it is an infinity of its sign
    scales *= 2.0 ** 30
    gq.w4_matvec(x, codes, scales, group, y)
    want, tol = want * 2.0 ** 30, tol * 2.0 ** 30
    top = float(torch.finfo(torch.float32).max)
    sure = (want.abs() + tol < top) | (want.abs() - tol > 2.0 * top)
    beyond = want.abs() > top
    want[beyond] *= float("inf")
    assert bool(sure[large].any()) and bool(beyond[sure].any())
    close(y[sure], want[sure], tol[sure])


# ---- callers ----------------------------------------------------------------------------------------------------------

def test_backward_refuses_what_is_no_matrix_like_the_other_calls():
    x, w = torch.zeros(2, 8), torch.zeros(8)
    with pytest.raises(TypeError):
        gq.rms_norm_backward(None, x, w, w, x, dweight_out=w)
    with pytest.raises(ValueError):
        gq.rms_norm_backward(torch.zeros(()), x, w, w, x, dweight_out=w)
