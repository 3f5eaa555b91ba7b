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


# ---- every shape of workgroup of the product over several steps and tiles -------------------------------------------

@gpu
@pytest.mark.parametrize("x_type,scale,group", [("bf16", "bf16", 128), ("bf16", "f32", 32), ("f16", "f32", 64), ("f16", "bf16", 32), ("i8", "f32", 32),
                                                ("i8", "bf16", 128), ("i8", "f32", 64)])
@pytest.mark.parametrize("m,rows,cols", [(1, 2000, 8300), (1, 16001, 2100), (2, 16001, 2100), (1, 30001, 4200), (8, 12300, 2500), (12, 2000, 8300), (12, 5000, 8300), (12, 9001, 8300),
                                         (16, 12000, 4200), (9, 17001, 2100), (30, 3000, 8300), (30, 5000, 8300), (30, 9001, 4200), (30, 12000, 4200), (32, 17001, 2100),
                                         (50, 3000, 4200), (50, 5000, 4200), (50, 9001, 4200), (64, 12000, 2100), (50, 17001, 2100), (130, 9001, 2100)])
def test_w4_matvec_over_several_steps(m, rows, cols, group, x_type, scale):
    """At least four steps of columns, the last one ragged, or more than one tile a workgroup, for each shape of workgroup."""
    g = torch.Generator(DEV).manual_seed(m * 7919 + rows * 31 + cols + group)
    q, codes, scales = device_weights(g, rows, cols, group, TYPES[scale])
    if x_type == "i8":
        x, xs = torch.randint(-128, 128, (m, cols), generator=g, device=DEV).to(torch.int8), 0.01 + torch.rand(m, generator=g, device=DEV)
    else:
        x, xs = (torch.randn(m, cols, generator=g, device=DEV) * 0.1).to(TYPES[x_type]), None
    y = L.Guarded((m, rows), torch.float32)
    gq.w4_matvec(x, codes, scales, group, y.t, x_scales=xs)
    close(y.t, *exact_matvec(x, xs, q, scales, group))
    assert y.intact()
    again = torch.empty_like(y.t)
    for _ in range(2):
        gq.w4_matvec(x, codes, scales, group, again, x_scales=xs)
        assert torch.equal(again, y.t)


# ---- the weight's gradient ------------------------------------------------------------------------------------------

# rows of fewer than eight columns, every team of waves, rows that are read twice; in bfloat16 and binary32
TEAMS = [5, 64, 512, 900, 1500, 2500, 5003, 7001, 8193, 12_000, 16_384, 16_385, 20_001, 32_768]


@gpu
@pytest.mark.parametrize("drops", [False, True])
@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("n", TEAMS)
def test_weight_gradient_of_many_rows_keeps_small_terms(n, name, drops):
    """One row of 2^24 and ones in all others: a sum in binary32 that met the large row first would lose the ones behind it."""
    t, rows = TYPES[name], 60_000 if n < 1000 else 8000 if n < 3000 else 4100 if n < 16_385 else 2600
    h = torch.ones(rows, n, dtype=t, device=DEV)
    dy, dx = torch.ones_like(h), torch.empty_like(h)
    dy[0] = 2.0 ** 24
    dw, one = torch.empty(n, device=DEV), torch.ones(rows, device=DEV)
    drop = gq.make_dropout(0.1, 5) if drops else None
    gq.rms_norm_backward(dy, h, torch.ones(n, dtype=t, device=DEV), one, dx, dweight_out=dw, drop=drop)
    want = torch.full((n,), 2.0 ** 24 + rows - 1, dtype=torch.float64)
    # h rstd and the products are exact; a part of the sum and the sum are rounded once each
    close(dw, want, 2 * U * want)


@gpu
@pytest.mark.parametrize("rows", [1, 300, 1000, 2100, 9000])
@pytest.mark.parametrize("n", TEAMS)
def test_weight_gradient_is_rounded_no_more_often_with_more_rows(n, rows):
    if rows * n > 40_000_000:
        rows = 40_000_000 // n
    g = torch.Generator(DEV).manual_seed(n + rows)
    h, dy = (torch.randn(rows, n, generator=g, device=DEV) for _ in range(2))
    rstd = (1.0 / torch.sqrt(h.double().square().mean(1) + 1e-5)).float()
    dw, again, dx = torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty_like(h)
    ws = torch.full((gq.rms_norm_workspace_bytes(rows, n),), 0xFF, dtype=torch.uint8, device=DEV)      # NaN where nothing is written
    w = torch.randn(n, generator=g, device=DEV)
    gq.rms_norm_backward(dy, h, w, rstd, dx, dweight_out=dw, workspace=ws)
    terms = dy.double() * h.double() * rstd.double()[:, None]
    # h rstd, a part, and the sum
    close(dw, terms.sum(0), 1.01 * U * (2 * terms.abs().sum(0) + terms.sum(0).abs()))
    gq.rms_norm_backward(dy, h, w, rstd, dx, dweight_out=again)
    assert torch.equal(again, dw)


# ---- rows that the registers do not hold, and the longest that they do: more rows than workgroups ---------------------

@gpu
@pytest.mark.parametrize("draws", [0, 16, 32])
@pytest.mark.parametrize("with_dsum", [False, True])
@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("n", [8200, 12_001, 16_384, 16_385, 20_001, 32_768])
def test_rms_norm_backward_of_many_long_rows(n, name, with_dsum, draws):
    rows, t = 1100 if name == "bf16" else 600, TYPES[name]
    g = torch.Generator(DEV).manual_seed(n + draws)
    h, dy, ds = (torch.randn(rows, n, generator=g, device=DEV).to(t) for _ in range(3))
    w = torch.randn(n, generator=g, device=DEV).to(t)
    ds = ds if with_dsum else None
    rstd = (1.0 / torch.sqrt(h.double().square().mean(1) + 1e-5)).float()
    make = lambda first: gq.make_dropout(0.25, L.SEED, 2, 8 * math.ceil(n / 8) * first, draws) if draws else None     # noqa: E731
    dx, dres, dw = L.Guarded((rows, n), t), L.Guarded((rows, n), t), L.Guarded((n,), torch.float32)
    gq.rms_norm_backward(dy, h, w, rstd, dx.t, dsum=ds, dres_out=dres.t if draws else None, dweight_out=dw.t, drop=make(0))
    assert dx.intact() and dres.intact() and dw.intact()
    for a, b in ((0, 3), (254, 260), (510, 516), (rows - 5, rows)):     # a few of the rows in 64 bits, and in a call of their own
        xh, gr = h[a:b].double() * rstd[a:b].double()[:, None], dy[a:b].double() * w.double()
        c, ca = (gr * xh).mean(1, keepdim=True), (gr * xh).abs().mean(1, keepdim=True)
        dh = rstd[a:b].double()[:, None] * (gr - xh * c)
        tol = U * rstd[a:b].double()[:, None] * (3 * gr.abs() + xh.abs() * (3 * c.abs() + 2 * ca) + 2 * (gr - xh * c).abs()) * 1.01
        if with_dsum:
            dh = ds[a:b].double() + dh
            tol = tol + U * (dh.abs() + tol)
        got = dres.t if draws else dx.t
        close(got[a:b], dh, tol + L.half_step(t) * (dh.abs() + tol) + L.least(t))
        px, pres = torch.empty(b - a, n, dtype=t, device=DEV), torch.empty(b - a, n, dtype=t, device=DEV)
        gq.rms_norm_backward(dy[a:b].clone(), h[a:b].clone(), w, rstd[a:b].clone(), px, dsum=None if ds is None else ds[a:b].clone(),
                             dres_out=pres if draws else None, drop=make(a))
        assert torch.equal(px, dx.t[a:b]) and (not draws or torch.equal(pres, dres.t[a:b]))
    terms = dy.double() * h.double() * rstd.double()[:, None]
    close(dw.t, terms.sum(0), 1.01 * U * (2 * terms.abs().sum(0) + terms.sum(0).abs()))
    again = torch.empty(n, device=DEV)
    if ds is not None:                                                # over dy and dsum
        gq.rms_norm_backward(dy, h, w, rstd, dy, dsum=ds, dres_out=ds if draws else None, dweight_out=again, drop=make(0))
        assert torch.equal(dy, dx.t) and (not draws or torch.equal(ds, dres.t)) and torch.equal(again, dw.t)


# ---- long launches of every type --------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows,n", [(4200, 4096), (4100, 4104), (4100, 4099), (1, 17_000_003)])
def test_long_dropouts_of_every_type(rows, n, name):
    t = TYPES[name]
    x = torch.randn(rows, n, device=DEV).to(t)
    res, whole, pitch = torch.randn(rows, n, device=DEV).to(t), L.Guarded((rows, n), t), 8 * math.ceil(n / 8)
    for bits in (32, 16):
        for r in (None, res):
            gq.dropout(x, gq.make_dropout(0.4, 9, 1, 16, bits), whole.t, residual=r)
            assert whole.intact()
            for a, b in ((0, 8), (rows // 2, rows // 2 + 8), (rows - 8, rows)) if rows > 1 else ((0, 8000), (8_000_000, 8_008_000), (n - 8003, n)):
                part = (slice(a, b), slice(0, n)) if rows > 1 else (slice(0, 1), slice(a, b))
                drop = gq.make_dropout(0.4, 9, 1, 16 + (pitch * a if rows > 1 else a), bits)
                k, by = L.kept(b - a if rows > 1 else 1, n if rows > 1 else b - a, drop)
                v = torch.where(k, x[part].double().cpu() * by, 0.0)
                want = v if r is None else r[part].double().cpu() + v
                close(whole.t[part], want, 2 * U * v.abs() + (U + L.half_step(t)) * (want.abs() + 2 * U * v.abs()) + L.least(t))


@gpu
@pytest.mark.parametrize("scale", ["f32", "bf16"])
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,cols", [(4200, 4096), (4100, 4104), (4100, 4099), (8200, 2047)])
def test_long_weights_of_every_type(rows, cols, group, name, scale):
    """Whole groups a row, and ragged ones; a few of the rows against the definition."""
    t, st, G = TYPES[name], TYPES[scale], -(-cols // group)
    w = (torch.randn(rows, cols, device=DEV) * 0.02).to(t)
    codes, scales, out = L.Guarded((rows, gq.w4_row_bytes(cols)), torch.uint8), L.Guarded((rows, G), st), L.Guarded((rows, cols), t)
    gq.group_quantize(w, group, codes.t, scales.t)
    gq.group_dequantize(codes.t, scales.t, group, out.t)
    assert codes.intact() and scales.intact() and out.intact()
    for a, b in ((0, 20), (rows // 2, rows // 2 + 20), (rows - 20, rows)):
        part = w[a:b].cpu()
        padded = torch.nn.functional.pad(part, (0, G * group - cols)).reshape(b - a, G, group)
        want = (padded.float().abs().amax(2) * torch.tensor(1.0 / 7.0)).to(st)
        assert torch.equal(scales.t[a:b].cpu(), want)
        s = L.per_column(want, cols, group)
        q = L.unpacked(codes.t[a:b], cols)
        assert torch.equal(q[:, :cols], (part.double() / s).round().clamp(-7, 7).long()) and not q[:, cols:].any()
        value = q[:, :cols].double() * s
        close(out.t[a:b], value, (U + L.half_step(t)) * value.abs() + L.least(t))


# ---- callers ----------------------------------------------------------------------------------------------------------

@gpu
def test_autograd_sees_what_is_written():
    """A tensor that autograd keeps for its backward pass and a call writes over: the backward pass refuses, as for torch's own operations."""
    z = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device=DEV)                     # noqa: E731
    drop, w = gq.make_dropout(0.1, 1), torch.ones(8, device=DEV)
    codes, scales = z(4, 16, t=torch.uint8), torch.ones(4, 1, device=DEV)
    gq.group_quantize(torch.randn(4, 8, device=DEV), 32, codes, scales)
    calls = {"dropout": lambda o: gq.dropout(z(4, 8), drop, o),
             "dropout over the residual": lambda o: gq.dropout(z(4, 8), drop, o, residual=o),
             "norm": lambda o: gq.rms_norm(z(4, 8), w, 1e-5, o),
             "sum": lambda o: gq.rms_norm(z(4, 8), w, 1e-5, z(4, 8), residual=o, sum_out=o),
             "backward": lambda o: gq.rms_norm_backward(z(4, 8), z(4, 8), w, z(4), o),
             "the residual's gradient": lambda o: gq.rms_norm_backward(z(4, 8), z(4, 8), w, z(4), z(4, 8), dres_out=o, drop=drop),
             "unfolded": lambda o: gq.group_dequantize(codes, scales, 32, o)}
    for what, call in calls.items():
        leaf = torch.randn(4, 8, device=DEV, requires_grad=True)
        kept = leaf * 2.0
        loss = (kept * kept).sum()
        call(kept.detach())                                           # shares memory and version with what autograd keeps
        with pytest.raises(RuntimeError, match="inplace"):
            loss.backward()
    vectors = {"rstd_out": lambda o: gq.rms_norm(z(4, 8), w, 1e-5, z(4, 8), rstd_out=o),
               "scales_out": lambda o: gq.rms_norm(z(4, 8), w, 1e-5, z(4, 8, t=torch.int8), scales_out=o),
               "product": lambda o: gq.w4_matvec(z(1, 8, t=torch.bfloat16), codes, scales, 32, o.view(1, 4)),
               "scales": lambda o: gq.group_quantize(z(4, 8), 32, codes, o.view(4, 1))}
    for what, call in vectors.items():
        o = z(4)
        before = o._version
        call(o)
        assert o._version == before + 1, what
    o, before = z(8), codes._version
    gq.rms_norm_backward(z(4, 8), z(4, 8), w, z(4), z(4, 8), dweight_out=o)
    assert o._version == 1
    gq.group_quantize(z(4, 8), 32, codes, scales)
    assert codes._version == before + 1
    x = z(4, 8)
    with pytest.raises(gq.GQError):                                   # a call that is refused has written nothing
        gq.rms_norm(z(4, 8), w, -1.0, x)
    assert x._version == 0 and w._version == 0
    with torch.inference_mode():                                      # such tensors have no version
        gq.dropout(z(4, 8), drop, z(4, 8))


def test_backward_refuses_what_is_no_matrix_like_the_other_calls():
    x, w = torch.zeros(2, 8), torch.zeros(8)
    with pytest.raises(TypeError):
        gq.rms_norm_backward(None, x, w, w, x, dweight_out=w)
    with pytest.raises(ValueError):
        gq.rms_norm_backward(torch.zeros(()), x, w, w, x, dweight_out=w)


# ---- as many elements as a call takes ---------------------------------------------------------------------------------

@gpu
def test_dropout_of_as_many_elements_as_a_matrix_may_have():
    """2^35 elements, in place: the last rows are those of a call on them alone."""
    rows, n, last = 1 << 19, 1 << 16, (1 << 19) - 8
    x = torch.ones(rows, n, dtype=torch.bfloat16, device=DEV)
    tail = torch.empty(8, n, dtype=x.dtype, device=DEV)
    gq.dropout(x[last:], gq.make_dropout(0.3, 9, index_base=n * last), tail)
    middle = torch.empty(8, n, dtype=x.dtype, device=DEV)
    gq.dropout(x[rows // 2 - 4:rows // 2 + 4], gq.make_dropout(0.3, 9, index_base=n * (rows // 2 - 4)), middle)
    gq.dropout(x, gq.make_dropout(0.3, 9), x)
    assert torch.equal(x[last:], tail) and torch.equal(x[rows // 2 - 4:rows // 2 + 4], middle)


@gpu
def test_weights_of_as_many_units_as_a_call_takes():
    """Short rows of binary32 weights, padded to a group of 128: 2^32 units of eight columns."""
    rows, cols, last = 1 << 28, 33, (1 << 28) - 8
    w = torch.empty(rows, cols, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(1))
    codes = torch.empty(rows, gq.w4_row_bytes(cols), dtype=torch.uint8, device=DEV)
    scales = torch.empty(rows, 1, device=DEV)
    gq.group_quantize(w, 128, codes, scales)
    tc, ts = torch.empty_like(codes[last:]), torch.empty_like(scales[last:])
    gq.group_quantize(w[last:].clone(), 128, tc, ts)
    assert torch.equal(codes[last:], tc) and torch.equal(scales[last:], ts)
