"""The layers around the gradient exchange (dropout, RMS norm, 4-bit weights and their product) against plain implementations in
64 bits.  Tolerances count roundings: u = 2^-24 for a binary32 step, half = finfo(t).eps / 2 for the rounding to an output's type."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2305_18627_amd as gq
from oracle import gq_oracle as O

gpu = pytest.mark.gpu
DEV = torch.device("cuda:0")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24
M32 = 0xFFFFFFFF
SEED = 0x1234567890ABCDEF


def half_step(t):
    return torch.finfo(t).eps / 2


def least(t):
    """What a result may be off where it is so small that the type's steps no longer shrink with it: half its smallest number."""
    return float(torch.finfo(t).smallest_normal) * float(torch.finfo(t).eps) / 2


def close(got, want, tol):
    """|got - want| <= tol wherever want is a number, and the same infinities and NaN."""
    got, want = got.detach().double().cpu(), want.double().cpu()
    tol = torch.as_tensor(tol, dtype=torch.float64).cpu().expand(want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])
    off = (got - want).abs()[fine] - tol[fine]
    assert not off.numel() or float(off.max()) <= 0.0, "off by %g over its tolerance" % float(off.max())


class Guarded:
    """A contiguous tensor with a pattern behind its last element that no call may change."""

    def __init__(self, shape, dtype):
        n = int(np.prod(shape))
        self.size = torch.empty(0, dtype=dtype).element_size()
        self.all = torch.full((n * self.size + 256,), 0x5A, dtype=torch.uint8, device=DEV)
        self.t = self.all[:n * self.size].view(dtype).view(shape)

    def intact(self):
        torch.cuda.synchronize()
        return bool((self.all[-256:] == 0x5A).all())


# ---- the random stream in plain numpy -------------------------------------------------------------------------------

def philox(call, worker, seed, domain=3):
    lo = np.uint64(M32)
    call = np.asarray(call, dtype=np.uint64)
    c = [call & lo, call >> np.uint64(32), np.full_like(call, worker), np.full_like(call, domain)]
    k = [seed & M32, seed >> 32]
    for _ in range(10):
        p, q = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & lo, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & lo]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return np.stack(c, -1).astype(np.uint32)


def kept(rows, n, drop):
    """(which elements are kept, their scale) by the definition in the header."""
    bits = drop.rng_bits or 32
    t = min(round(drop.p * 2 ** bits), 2 ** bits - 1)                # Python's round: ties to even
    pitch = 8 * math.ceil(n / 8)
    g = drop.index_base + np.arange(rows * pitch, dtype=np.int64)
    per = 4 if bits == 32 else 8
    first = int(drop.index_base) // per
    words = philox(np.arange(first, first + -(-rows * pitch // per) + 1, dtype=np.uint64), drop.worker, drop.seed)
    at = g - per * first
    if bits == 32:
        r = words.reshape(-1)[at]
    else:
        w = words[at // 8, (at % 8) // 2]
        r = np.where(at % 2 == 0, w & 0xFFFF, w >> 16)
    k = (r >= t).reshape(rows, pitch)[:, :n]
    return torch.from_numpy(np.ascontiguousarray(k)), 2.0 ** bits / (2.0 ** bits - t)


def test_the_plain_generator_is_the_oracles():
    for call, worker in ((0, 0), (5, 3), (1 << 40, 7), ((1 << 61) + 12345, 0xFFFFFFFF)):
        want = O.philox4x32([call & M32, call >> 32, worker, 3], [SEED & M32, SEED >> 32])
        assert np.array_equal(philox([call], worker, SEED)[0], np.asarray(want, dtype=np.uint32))


# ---- refusals, on the CPU -------------------------------------------------------------------------------------------

def test_refusals_of_the_c_abi_need_no_device():
    lib, I = gq.lib(), gq.GQ_ERR_INVALID_ARG
    ok, odd = C.c_void_p(0x1000), C.c_void_p(0x1008)
    D = gq.make_dropout
    ref = lambda d: C.byref(d) if d is not None else None                                    # noqa: E731
    dr = lambda x=ok, res=None, rows=2, n=8, t=1, d=D(0.1, 1), out=ok: lib.gq_dropout(x, res, rows, n, t, ref(d), out, None)  # noqa: E731
    for bad in (D(-0.1, 1), D(1.0, 1), D(float("nan"), 1), D(0.1, 1, rng_bits=8), D(0.1, 1, index_base=-4), D(0.1, 1, index_base=2),
                D(0.1, 1, index_base=4, rng_bits=16), D(0.1, 1, index_base=(1 << 63) - 8), None):
        assert dr(d=bad) == I
    assert dr(x=odd) == I and dr(out=odd) == I and dr(res=odd) == I and dr(x=None) == I and dr(out=None) == I
    assert dr(rows=-1) == I and dr(n=-1) == I and dr(t=3) == I and dr(t=9) == I and dr(t=-1) == I and dr(rows=1 << 31) == I
    assert dr(rows=1 << 20, n=1 << 20) == I
    assert dr(rows=0, x=None, out=None) == gq.GQ_OK and dr(n=0) == gq.GQ_OK

    def norm(x=ok, res=None, rows=2, n=8, t=1, w=ok, wt=1, eps=1e-5, d=None, s=None, out=C.c_void_p(0x2000), ot=1, sc=None, rstd=None):
        return lib.gq_rms_norm(x, res, rows, n, t, w, wt, eps, ref(d), s, out, ot, sc, rstd, None)
    for eps in (0.0, -1.0, float("inf"), float("nan")):
        assert norm(eps=eps) == I
    assert norm(t=3) == I and norm(wt=2) == I and norm(t=2, wt=1) == I and norm(ot=0) == I and norm(ot=2) == I and norm(ot=7) == I
    assert norm(ot=3) == I and norm(ot=4) == I and norm(sc=ok) == I                        # scales with 8 bits, and only then
    assert norm(x=odd) == I and norm(w=odd) == I and norm(out=odd) == I and norm(res=odd) == I and norm(s=odd) == I
    assert norm(s=C.c_void_p(0x2000)) == I                                                 # sum and out in one place
    assert norm(ot=3, sc=ok, out=ok) == I and norm(ot=4, sc=ok, res=C.c_void_p(0x2000)) == I     # 8 bits over 16
    assert norm(rstd=C.c_void_p(0x1002)) == I and norm(ot=3, sc=C.c_void_p(0x1002)) == I
    assert norm(d=D(1.5, 1)) == I and norm(rows=-1) == I
    assert norm(n=gq.GQ_RMS_NORM_MAX_N + 1) == gq.GQ_ERR_UNSUPPORTED
    assert norm(rows=0) == gq.GQ_OK and norm(n=0) == gq.GQ_OK

    def back(dy=ok, h=ok, ds=None, rows=2, n=8, t=1, w=ok, wt=1, rstd=ok, d=None, dres=None, dx=ok, dw=None, ws=None, wsb=0):
        return lib.gq_rms_norm_backward(dy, h, ds, rows, n, t, w, wt, rstd, ref(d), dres, dx, dw, ws, wsb, None)
    assert back(dres=ok) == I                                                              # without drop it is dx_out
    assert back(d=D(0.1, 1), dres=ok, dx=ok) == I and back(dy=odd) == I and back(h=None) == I and back(rstd=None) == I and back(dx=None) == I
    assert back(ds=odd) == I and back(t=4) == I and back(wt=2) == I and back(dw=odd, ws=ok, wsb=1 << 20) == I
    assert back(dw=ok) == gq.GQ_ERR_WORKSPACE and back(dw=ok, ws=ok, wsb=8) == gq.GQ_ERR_WORKSPACE
    assert back(dw=ok, ws=odd, wsb=1 << 20) == gq.GQ_ERR_WORKSPACE
    assert back(n=gq.GQ_RMS_NORM_MAX_N + 1) == gq.GQ_ERR_UNSUPPORTED
    assert back(rows=0) == gq.GQ_OK and back(n=0, dw=ok) == gq.GQ_OK
    assert gq.rms_norm_workspace_bytes(-1, 8) == 0 and gq.rms_norm_workspace_bytes(8, gq.GQ_RMS_NORM_MAX_N + 1) == 0
    assert gq.rms_norm_workspace_bytes(0, 8) >= 32 and gq.rms_norm_workspace_bytes(1 << 20, 4096) <= 1 << 25

    assert [gq.w4_row_bytes(c) for c in (-1, 0, 1, 32, 33, 4096)] == [0, 0, 16, 16, 32, 2048]
    gqz = lambda w=ok, rows=2, cols=40, t=1, g=32, c=ok, s=ok, st=0: lib.gq_group_quantize(w, rows, cols, t, g, c, s, st, None)  # noqa: E731
    gdq = lambda c=ok, s=ok, st=0, rows=2, cols=40, g=32, o=ok, t=1: lib.gq_group_dequantize(c, s, st, rows, cols, g, o, t, None)  # noqa: E731
    for f in (gqz, gdq):
        assert f(g=16) == I and f(g=0) == I and f(g=256) == I and f(t=3) == I and f(st=2) == I and f(st=3) == I and f(rows=-1) == I
        assert f(c=odd) == I and f(s=odd) == I and f(cols=-1) == I and f(rows=0) == gq.GQ_OK and f(cols=0) == gq.GQ_OK
    assert gqz(w=odd) == I and gqz(w=None) == I and gdq(o=odd) == I and gdq(o=None) == I

    def mv(x=ok, xs=None, m=2, xt=1, c=ok, s=ok, st=0, rows=4, cols=40, g=32, b=None, y=ok, yt=1):
        return lib.gq_w4_matvec(x, xs, m, xt, c, s, st, rows, cols, g, b, y, yt, None)
    assert mv(xt=0) == I and mv(xt=4) == I and mv(yt=3) == I and mv(xt=3) == I and mv(xs=ok) == I and mv(g=48) == I and mv(st=2) == I
    assert mv(x=odd) == I and mv(c=odd) == I and mv(s=odd) == I and mv(y=odd) == I and mv(b=odd) == I and mv(xt=3, xs=C.c_void_p(0x1002)) == I
    assert mv(m=-1) == I and mv(rows=-1) == I and mv(cols=-1) == I and mv(m=1 << 31) == I and mv(m=(1 << 20) + 1) == I
    assert mv(rows=(1 << 30) + 1) == I and mv(cols=(1 << 24) + 1) == I
    assert mv(m=0) == gq.GQ_OK and mv(rows=0) == gq.GQ_OK


def test_refusals_of_the_binding_need_no_device():
    x, w, d = torch.zeros(2, 8), torch.zeros(8), gq.make_dropout(0.1, 1)
    c, s = torch.zeros(2, 16, dtype=torch.uint8), torch.zeros(2, 1)
    for call in (lambda: gq.dropout(x, d, x), lambda: gq.rms_norm(x, w, 1e-5, x), lambda: gq.rms_norm_backward(x, x, w, w, x),
                 lambda: gq.rms_norm_backward(x, x, w, w, x, dweight_out=w),
                 lambda: gq.group_quantize(x, 32, c, s), lambda: gq.group_dequantize(c, s, 32, x), lambda: gq.w4_matvec(x, c, s, 32, x)):
        with pytest.raises(ValueError):
            call()
    for bad in (gq.make_params(0, 7), 0.1, b"x" * 32):
        with pytest.raises(TypeError):
            gq.dropout(x, bad, x)
        with pytest.raises(TypeError):
            gq.rms_norm(x, w, 1e-5, x, drop=bad)
    with pytest.raises(TypeError):
        gq.dropout(None, d, x)


@gpu
def test_refusals_of_the_binding():
    z = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device=DEV)                     # noqa: E731
    x, w, d = z(4, 8), z(8), gq.make_dropout(0.1, 1)
    c, s, u8 = z(4, 16, t=torch.uint8), z(4, 1), torch.uint8
    for call in (lambda: gq.dropout(x, d, z(4, 7)), lambda: gq.dropout(x, d, z(4, 8, t=torch.bfloat16)), lambda: gq.dropout(x.t(), d, x.t()),
                 lambda: gq.dropout(x, d, x, residual=z(3, 8)), lambda: gq.dropout(x, d, torch.zeros(4, 8)),
                 lambda: gq.dropout(z(4, 8, t=torch.float64), d, z(4, 8, t=torch.float64)), lambda: gq.dropout(z(8)[0], d, z(8)[0]),
                 lambda: gq.rms_norm(x, z(7), 1e-5, x), lambda: gq.rms_norm(x, w, 1e-5, z(4, 7)),
                 lambda: gq.rms_norm(x, w, 1e-5, z(4, 8, t=torch.int8), scales_out=z(3)), lambda: gq.rms_norm(x, w, 1e-5, x, rstd_out=z(5)),
                 lambda: gq.rms_norm_backward(x, z(4, 7), w, z(4), x), lambda: gq.rms_norm_backward(x, x, w, z(3), x),
                 lambda: gq.rms_norm_backward(x, x, w, z(4), z(4, 8), dweight_out=z(7)),
                 lambda: gq.group_quantize(x, 32, z(4, 15, t=u8), s), lambda: gq.group_quantize(x, 32, z(3, 16, t=u8), z(3, 1)),
                 lambda: gq.group_quantize(x, 32, c, z(4, 2)), lambda: gq.group_quantize(x, 0, c, s), lambda: gq.group_quantize(x, -32, c, s),
                 lambda: gq.group_quantize(x, 1 << 40, c, s), lambda: gq.group_dequantize(c, s, 32, z(3, 8)),
                 lambda: gq.w4_matvec(z(2, 8, t=torch.bfloat16), c, s, 32, z(2, 5)), lambda: gq.w4_matvec(z(2, 8, t=torch.bfloat16), c, s, 32, z(3, 4)),
                 lambda: gq.w4_matvec(z(2, 8, t=torch.bfloat16), c, s, 32, z(2, 4), bias=z(4, t=torch.bfloat16)),
                 lambda: gq.w4_matvec(z(2, 8, t=torch.int8), c, s, 32, z(2, 4), x_scales=z(3))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: gq.dropout(z(4, 8, t=torch.int8), d, z(4, 8, t=torch.int8)), lambda: gq.rms_norm(x, w, 0.0, z(4, 8)),
                 lambda: gq.rms_norm(x, w, 1e-5, z(4, 8, t=torch.int8)), lambda: gq.rms_norm(x, z(8, t=torch.float16), 1e-5, z(4, 8)),
                 lambda: gq.rms_norm(x, w, 1e-5, x, sum_out=x), lambda: gq.rms_norm_backward(x, x, w, z(4), z(4, 8), dres_out=z(4, 8)),
                 lambda: gq.group_quantize(x, 16, c, s), lambda: gq.w4_matvec(x, c, s, 32, z(4, 4)),
                 lambda: gq.w4_matvec(z(4, 8, t=torch.int8), c, s, 32, z(4, 4)),
                 lambda: gq.rms_norm(z(1, 32769), z(32769), 1e-5, z(1, 32769)),
                 lambda: gq.rms_norm(z(5)[1:].view(1, 4), z(4), 1e-5, z(1, 4))):              # not 16-byte aligned
        with pytest.raises(gq.GQError):
            call()
    torch.cuda.synchronize()


# ---- dropout --------------------------------------------------------------------------------------------------------

def randn(g, *shape, std=1.0, t=torch.float32):
    return (torch.randn(*shape, generator=g) * std).to(t)


SHAPES = [(1, 1), (3, 7), (2, 8), (5, 9), (64, 64), (7, 511), (3, 2048), (1, 100_003), (37, 1000)]


@gpu
@pytest.mark.parametrize("bits", [32, 16])
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("rows,n", SHAPES)
def test_dropout(rows, n, name, bits):
    t = TYPES[name]
    g = torch.Generator().manual_seed(rows * 1000 + n)
    x, res = randn(g, rows, n, t=t), randn(g, rows, n, std=3.0, t=t)
    drop = gq.make_dropout(0.3, SEED, worker=5, index_base=(1 << 34) + 24, rng_bits=bits)
    k, by = kept(rows, n, drop)
    x[~k] = float("nan")                                             # what is dropped is gone, whatever it held
    if n > 1:
        x[0, 1 if k[0, 1] else 0] = float("inf") if k[0, 1] else x[0, 0]
    v = torch.where(k, x.double() * by, 0.0)
    for r in (None, res):
        want = v if r is None else r.double() + v
        out = Guarded((rows, n), t)
        gq.dropout(x.to(DEV), drop, out.t, None if r is None else r.to(DEV))
        # the scale and its product: two roundings of v; the sum and the output: one each
        close(out.t, want, 2 * U * v.abs() + (U + half_step(t)) * (want.abs() + 2 * U * v.abs()) + least(t))
        assert out.intact()
    xd, rd = x.to(DEV), res.to(DEV)
    gq.dropout(xd, drop, xd, rd)                                     # in place of x, and of the residual
    assert torch.equal(xd.view(torch.uint8), out.t.view(torch.uint8))
    gq.dropout(x.to(DEV), drop, rd, rd)
    assert torch.equal(rd.view(torch.uint8), out.t.view(torch.uint8))


@gpu
@pytest.mark.parametrize("bits", [32, 16])
@pytest.mark.parametrize("p", [0.0, 1e-12, 0.5, 0.999999999999])
def test_dropout_probabilities_at_their_ends(p, bits):
    x = torch.ones(16, 4096, device=DEV)
    out = torch.empty_like(x)
    drop = gq.make_dropout(p, 3, rng_bits=bits)
    gq.dropout(x, drop, out)
    k, by = kept(16, 4096, drop)
    assert torch.equal(out.cpu() != 0, k)
    close(out, torch.where(k, by, 0.0).double(), 2 * U * by)


@gpu
@pytest.mark.parametrize("bits", [32, 16])
@pytest.mark.parametrize("n", [5, 64])
def test_dropout_of_a_matrix_cut_between_rows(n, bits):
    x = torch.randn(50, n, device=DEV)
    whole, parts = torch.empty_like(x), torch.empty_like(x)
    gq.dropout(x, gq.make_dropout(0.4, 9, 1, 16, bits), whole)
    for a, b in ((0, 20), (20, 50)):
        piece = torch.empty(b - a, n, device=DEV)
        gq.dropout(x[a:b].clone(), gq.make_dropout(0.4, 9, 1, 16 + 8 * math.ceil(n / 8) * a, bits), piece)
        parts[a:b] = piece
    assert torch.equal(whole, parts)
    other = torch.empty_like(x)
    gq.dropout(x, gq.make_dropout(0.4, 9, 2, 16, bits), other)
    assert not torch.equal(whole, other)                             # another worker draws on its own


@gpu
@pytest.mark.parametrize("rows,n", [(4100, 4104), (4100, 4099), (1, 17_000_003)])
def test_long_launches_equal_their_parts(rows, n):
    """Dropout and 4-bit weights of more elements than a short launch has: whole rows against calls on some of them."""
    x = torch.randn(rows, n, device=DEV, dtype=torch.bfloat16)
    whole = torch.empty_like(x)
    pitch = 8 * math.ceil(n / 8)
    for bits in (32, 16):
        gq.dropout(x, gq.make_dropout(0.4, 9, 1, 16, bits), whole, residual=x)
        if rows == 1:                                                 # whole units: one row of the stream
            for a, b in ((0, 8000), (8_000_000, 8_100_000), (17_000_000 - 8000, n)):
                part = torch.empty(1, b - a, device=DEV, dtype=x.dtype)
                gq.dropout(x[:, a:b].clone(), gq.make_dropout(0.4, 9, 1, 16 + a, bits), part, residual=x[:, a:b].clone())
                assert torch.equal(part, whole[:, a:b])
        else:
            for a, b in ((0, 50), (2040, 2100), (rows - 30, rows)):
                part = torch.empty(b - a, n, device=DEV, dtype=x.dtype)
                gq.dropout(x[a:b].clone(), gq.make_dropout(0.4, 9, 1, 16 + pitch * a, bits), part, residual=x[a:b].clone())
                assert torch.equal(part, whole[a:b])
    if rows == 1:
        return
    for group in (32, 64, 128):
        G, st = -(-n // group), torch.bfloat16
        codes, scales = Guarded((rows, gq.w4_row_bytes(n)), torch.uint8), Guarded((rows, G), st)
        gq.group_quantize(x, group, codes.t, scales.t)
        gq.group_dequantize(codes.t, scales.t, group, whole)
        for a, b in ((0, 50), (2040, 2100), (rows - 30, rows)):
            pc, ps, pv = torch.empty(b - a, gq.w4_row_bytes(n), dtype=torch.uint8, device=DEV), torch.empty(b - a, G, dtype=st, device=DEV), torch.empty(b - a, n, device=DEV, dtype=x.dtype)
            gq.group_quantize(x[a:b].clone(), group, pc, ps)
            gq.group_dequantize(pc, ps, group, pv)
            assert torch.equal(pc, codes.t[a:b]) and torch.equal(ps, scales.t[a:b]) and torch.equal(pv, whole[a:b])
        assert codes.intact() and scales.intact()


# ---- RMS norm -------------------------------------------------------------------------------------------------------

NS = [1, 7, 8, 65, 512, 1000, 2047, 2048, 2049, 4096, 5003, 8192, 8193, 16384, 20001, 32768]


def norm_inputs(rows, n, t, wt, seed=1):
    g = torch.Generator().manual_seed(seed * 100_000 + rows * 1000 + n)
    return randn(g, rows, n, t=t), randn(g, rows, n, std=3.0, t=t), (1.0 + randn(g, n, std=0.3)).to(wt)


def plain_norm(x, res, w, eps, drop):
    """(h, its tolerance, rstd, its relative tolerance, y, its tolerance before the last rounding) in 64 bits."""
    v = x.double()
    dh = torch.zeros_like(v)
    if drop is not None:
        k, by = kept(*x.shape, drop)
        v = torch.where(k, v * by, 0.0)
        dh = 2 * U * v.abs()                                          # the scale and the product
    h = v
    if res is not None:
        h = res.double() + v
        dh = dh + U * (h.abs() + dh)                                  # the sum
    ss = (h * h).sum(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(ss / x.shape[1] + eps)
    # |d rstd| / rstd <= sum |h| |dh| / sum h^2 to first order (doubled for the rest), and its own rounding
    rel = 2 * (h.abs() * dh).sum(1, keepdim=True) / ss.clamp_min(1e-300) + U
    y = h * rstd * w.double()
    dy = dh * rstd * w.double().abs() + y.abs() * (rel + 2 * U)       # two products
    return h, dh, rstd, rel, y, 1.01 * dy


@gpu
@pytest.mark.parametrize("name,weight", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("rows", [1, 5])
@pytest.mark.parametrize("n", NS)
def test_rms_norm(n, rows, name, weight):
    t, wt = TYPES[name], TYPES[weight]
    x, res, w = norm_inputs(rows, n, t, wt)
    for r, drop in ((None, None), (res, None), (res, gq.make_dropout(0.25, SEED, 2, 8, 32)), (None, gq.make_dropout(0.6, SEED, 2, 16, 16))):
        h, dh, rstd, rel, y, dy = plain_norm(x, r, w, 1e-5, drop)
        s, out, rs = Guarded((rows, n), t), Guarded((rows, n), t), Guarded((rows,), torch.float32)
        xd, rd, wd = x.to(DEV), None if r is None else r.to(DEV), w.to(DEV)
        gq.rms_norm(xd, wd, 1e-5, out.t, residual=rd, sum_out=s.t, rstd_out=rs.t, drop=drop)
        close(s.t, h, dh + half_step(t) * (h.abs() + dh) + least(t))
        close(rs.t, rstd[:, 0], (rstd * rel)[:, 0])
        close(out.t, y, dy + half_step(t) * (y.abs() + dy) + least(t))
        assert s.intact() and out.intact() and rs.intact()
        bare = torch.empty_like(xd)                                   # without the outputs that may be left out
        gq.rms_norm(xd, wd, 1e-5, bare, residual=rd, drop=drop)
        assert torch.equal(bare, out.t)
        if rd is not None:                                            # the residual stream updated in place, out over x
            gq.rms_norm(xd, wd, 1e-5, xd, residual=rd, sum_out=rd, drop=drop)
            assert torch.equal(xd, out.t) and torch.equal(rd, s.t)
        else:
            gq.rms_norm(xd, wd, 1e-5, bare, sum_out=xd, drop=drop)
            assert torch.equal(bare, out.t) and torch.equal(xd, s.t)


def e4m3_half_step(v):
    return torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 4)


@gpu
@pytest.mark.parametrize("kind", ["i8", "e4m3"])
@pytest.mark.parametrize("name,weight", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("n", NS)
def test_rms_norm_in_8_bits(n, name, weight, kind):
    t, rows = TYPES[name], 4
    x, res, w = norm_inputs(rows, n, t, TYPES[weight], seed=2)
    x[1], res[1] = 0.0, 0.0                                           # a row of zeros
    drop = gq.make_dropout(0.1, SEED)
    h, dh, rstd, rel, y, dy = plain_norm(x, res, w, 1e-5, drop)
    top, ot = (127.0, torch.int8) if kind == "i8" else (448.0, torch.float8_e4m3fn)
    s, out, sc = Guarded((rows, n), t), Guarded((rows, n), ot), Guarded((rows,), torch.float32)
    gq.rms_norm(x.to(DEV), w.to(DEV), 1e-5, out.t, residual=res.to(DEV), sum_out=s.t, scales_out=sc.t, drop=drop)
    assert s.intact() and out.intact() and sc.intact()
    want = y.abs().amax(1) / top
    close(sc.t, want, dy.amax(1) / top + 2 * U * want + 2.0 ** -149)
    scale = sc.t.double().cpu()[:, None]
    assert float(scale[1]) == 0.0 and not out.t.float()[1].any()
    got = out.t.float().double().cpu()
    live = scale[:, 0] > 0
    v, off = (y / scale)[live], (dy / scale)[live] + 3 * U * (y / scale)[live].abs()      # y inv: the quotient 1 / scale, the product
    close(got[live], v.clamp(-top, top), off + (0.5 if kind == "i8" else e4m3_half_step(v.abs() + off)))
    assert float(got[live].abs().amax(1).min()) == top


@gpu
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("n", [2049, 2500, 4096, 5003, 6144, 6200, 8192])
def test_rms_norm_of_many_rows(n, name):
    """Above 256 rows other teams of waves take rows of these lengths."""
    rows, t = 259, TYPES[name]
    x, res, w = norm_inputs(rows, n, t, t, seed=6)
    drop = gq.make_dropout(0.25, SEED, 2, 8, 32)
    h, dh, rstd, rel, y, dy = plain_norm(x, res, w, 1e-5, drop)
    s, out, rs, codes = Guarded((rows, n), t), Guarded((rows, n), t), Guarded((rows,), torch.float32), Guarded((rows, n), torch.int8)
    xd, rd, wd = x.to(DEV), res.to(DEV), w.to(DEV)
    sc = torch.empty(rows, device=DEV)
    gq.rms_norm(xd, wd, 1e-5, codes.t, residual=rd, scales_out=sc, drop=drop)
    gq.rms_norm(xd, wd, 1e-5, out.t, residual=rd, sum_out=s.t, rstd_out=rs.t, drop=drop)
    close(s.t, h, dh + half_step(t) * (h.abs() + dh) + least(t))
    close(rs.t, rstd[:, 0], (rstd * rel)[:, 0])
    close(out.t, y, dy + half_step(t) * (y.abs() + dy) + least(t))
    want = y.abs().amax(1) / 127.0
    close(sc, want, dy.amax(1) / 127.0 + 2 * U * want)
    scale = sc.double().cpu()[:, None]
    close(codes.t, (y / scale).clamp(-127, 127), dy / scale + 3 * U * (y / scale).abs() + 0.5)
    assert s.intact() and out.intact() and rs.intact() and codes.intact()
    gq.rms_norm(xd, wd, 1e-5, xd, residual=rd, sum_out=rd, drop=drop)
    assert torch.equal(xd, out.t) and torch.equal(rd, s.t)


@gpu
@pytest.mark.parametrize("kind", ["i8", "e4m3"])
def test_rms_norm_rows_that_are_not_finite_or_hardly_anything(kind):
    ot, n = (torch.int8 if kind == "i8" else torch.float8_e4m3fn), 300
    x = torch.randn(6, n)
    x[0, 17], x[1, 299], x[2, 5] = float("nan"), float("inf"), float("-inf")
    x[3] *= 1e-42                                                     # subnormal, under an eps that is large beside it
    x[4] *= 1e25                                                      # its squares are beyond binary32
    w = torch.ones(n)
    out, sc, y = torch.empty(6, n, dtype=ot, device=DEV), torch.empty(6, device=DEV), torch.empty(6, n, device=DEV)
    gq.rms_norm(x.to(DEV), w.to(DEV), 1e-5, out, scales_out=sc)
    gq.rms_norm(x.to(DEV), w.to(DEV), 1e-5, y)
    assert torch.isnan(sc[:3]).all() and not out[:3].float().any()
    assert float(sc[3]) == 0.0 and not out[3].float().any()           # 1 / scale is beyond binary32
    assert torch.isfinite(sc[3:]).all() and torch.isfinite(y[3:]).all()
    want = x[3:].double() / torch.sqrt(x[3:].double().square().mean(1, keepdim=True) + 1e-5)
    close(y[3:], want, 4 * U * want.abs() + 2.0 ** -149)
    close(sc[4:], want[1:].abs().amax(1) / (127.0 if kind == "i8" else 448.0), 6 * U)
    assert torch.isnan(y[0]).all() and torch.isnan(y[1, 299]) and not y[1, :299].any()


@gpu
@pytest.mark.parametrize("name,weight", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("rows", [1, 5, 300])
@pytest.mark.parametrize("n", NS)
def test_rms_norm_backward(n, rows, name, weight):
    if rows * n > 3_000_000:
        rows = 91
    t, wt = TYPES[name], TYPES[weight]
    h, dsum, w = norm_inputs(rows, n, t, wt, seed=3)
    dy = norm_inputs(rows, n, t, wt, seed=4)[0]
    rstd = (1.0 / torch.sqrt(h.double().square().mean(1) + 1e-5)).float()
    for ds, drop in ((None, None), (dsum, None), (dsum, gq.make_dropout(0.25, SEED, 2, 8, 32)), (None, gq.make_dropout(0.6, SEED, 2, 16, 16))):
        xh, g = h.double() * rstd.double()[:, None], dy.double() * w.double()
        c, ca = (g * xh).mean(1, keepdim=True), (g * xh).abs().mean(1, keepdim=True)
        dh = rstd.double()[:, None] * (g - xh * c)
        # g, xh, their part in c, c, xh c, the difference, the product with rstd: one rounding each
        tol = U * rstd.double()[:, None] * (3 * g.abs() + xh.abs() * (3 * c.abs() + 2 * ca) + 2 * (g - xh * c).abs()) * 1.01
        if ds is not None:
            dh = ds.double() + dh
            tol = tol + U * (dh.abs() + tol)
        dx, dres, dw = Guarded((rows, n), t), Guarded((rows, n), t), Guarded((n,), torch.float32)
        yd, hd, sd = dy.to(DEV), h.to(DEV), None if ds is None else ds.to(DEV)
        args = dict(dsum=sd, drop=drop)
        gq.rms_norm_backward(yd, hd, w.to(DEV), rstd.to(DEV), dx.t, dres_out=dres.t if drop else None, dweight_out=dw.t, **args)
        res_tol = tol + half_step(t) * (dh.abs() + tol) + least(t)
        if drop is None:
            close(dx.t, dh, res_tol)
        else:
            k, by = kept(rows, n, drop)
            v, dv = torch.where(k, dh * by, 0.0), torch.where(k, tol * by + 2 * U * (dh * by).abs(), 0.0)
            close(dres.t, dh, res_tol)
            close(dx.t, v, dv + half_step(t) * (v.abs() + dv) + least(t))
        # xh and the product, then a sum of `rows` terms in binary32
        close(dw.t, (dy.double() * xh).sum(0), (rows + 3) * U * (dy.double() * xh).abs().sum(0) + 2.0 ** -149)
        assert dx.intact() and dres.intact() and dw.intact()
        bare = torch.empty_like(yd)                                   # the weight's gradient and the residual's left out
        gq.rms_norm_backward(yd, hd, w.to(DEV), rstd.to(DEV), bare, **args)
        assert torch.equal(bare, dx.t)
        again, twice = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        if sd is not None and drop is not None:                       # over dy, and over dsum
            gq.rms_norm_backward(yd, hd, w.to(DEV), rstd.to(DEV), yd, dsum=sd, dres_out=sd, dweight_out=again, drop=drop)
            assert torch.equal(yd, dx.t) and torch.equal(sd, dres.t) and torch.equal(again, dw.t)
        elif sd is not None:
            gq.rms_norm_backward(yd, hd, w.to(DEV), rstd.to(DEV), sd, dsum=sd, dweight_out=twice)
            assert torch.equal(sd, dx.t) and torch.equal(twice, dw.t)


@gpu
@pytest.mark.parametrize("draws", [0, 16, 32])
@pytest.mark.parametrize("n", [5, 136, 900, 1500, 2500, 5003, 7001])
def test_rms_norm_backward_of_many_rows(n, draws):
    """More rows than a workgroup's first: each row alone against the same call on some of the rows, the weight's gradient against 64 bits."""
    rows = 8300 if n < 1000 else 2101
    g = torch.Generator().manual_seed(n)
    dev = lambda v: v.to(DEV)                                         # noqa: E731
    h, dy, ds, w = (dev(randn(g, *s, t=torch.bfloat16)) for s in ((rows, n), (rows, n), (rows, n), (n,)))
    rstd = (1.0 / torch.sqrt(h.double().square().mean(1) + 1e-5)).float()
    make = lambda first: gq.make_dropout(0.25, SEED, 2, 8 * math.ceil(n / 8) * first, draws) if draws else None     # noqa: E731
    dx, dres, dw = torch.empty_like(h), torch.empty_like(h), torch.empty(n, device=DEV)
    gq.rms_norm_backward(dy, h, w, rstd, dx, dsum=ds, dres_out=dres if draws else None, dweight_out=dw, drop=make(0))
    for a, b in ((0, 100), (700, 1100), (rows - 61, rows)):
        px, pres = torch.empty(b - a, n, dtype=h.dtype, device=DEV), torch.empty(b - a, n, dtype=h.dtype, device=DEV)
        cut = [v[a:b].clone() for v in (dy, h, ds, rstd)]
        gq.rms_norm_backward(cut[0], cut[1], w, cut[3], px, dsum=cut[2], dres_out=pres if draws else None, drop=make(a))
        assert torch.equal(px, dx[a:b]) and (not draws or torch.equal(pres, dres[a:b]))
    terms = dy.double() * h.double() * rstd.double()[:, None]
    # 512 or 256 parts of at most rows / 256 + 1 terms in turn, then 16 slices of 32 parts: that many roundings at most
    close(dw, terms.sum(0), (rows // 256 + 2 + 32 + 16 + 3) * U * terms.abs().sum(0))


@gpu
def test_rms_norm_backward_of_no_rows_clears_the_weights_gradient():
    dw = torch.full((40,), 7.0, device=DEV)
    e = torch.empty(0, 40, device=DEV)
    gq.rms_norm_backward(e, e, torch.ones(40, device=DEV), torch.empty(0, device=DEV), e, dweight_out=dw)
    assert not dw.any()


@gpu
@pytest.mark.parametrize("bits", [0, 32, 16])
@pytest.mark.parametrize("n", [9, 130, 2050])
def test_gradients_against_differences(n, bits):
    """x, residual and weight moved along a direction: the change of sum(dy y) + sum(ds h) in 64 bits against the gradients."""
    rows, eps = 6, 1e-3
    g = torch.Generator().manual_seed(n + bits)
    x, res, w, dy, ds = (randn(g, *s) for s in ((rows, n), (rows, n), (n,), (rows, n), (rows, n)))
    drop = gq.make_dropout(0.3, 77, 1, 0, bits) if bits else None
    dev = lambda v: v.to(DEV)                                         # noqa: E731
    h, y, rstd = torch.empty(rows, n, device=DEV), torch.empty(rows, n, device=DEV), torch.empty(rows, device=DEV)
    gq.rms_norm(dev(x), dev(w), eps, y, residual=dev(res), sum_out=h, rstd_out=rstd, drop=drop)
    dx, dres, dw = torch.empty(rows, n, device=DEV), torch.empty(rows, n, device=DEV), torch.empty(n, device=DEV)
    gq.rms_norm_backward(dev(dy), h, dev(w), rstd, dx, dsum=dev(ds), dres_out=dres if drop else None, dweight_out=dw, drop=drop)
    k, by = kept(rows, n, drop) if drop else (torch.ones(rows, n, dtype=torch.bool), 1.0)

    def loss(x, res, w):
        h = res + torch.where(k, x * by, 0.0)
        return float((dy.double() * (h / torch.sqrt(h.square().mean(1, keepdim=True) + eps) * w) + ds.double() * h).sum())
    at = [x.double(), res.double(), w.double()]
    for i, grad in enumerate((dx, dres if drop else dx, dw)):
        d = torch.randn(at[i].shape, generator=g, dtype=torch.float64)
        step = 1e-4
        up, down = ([a + s * d if j == i else a for j, a in enumerate(at)] for s in (step, -step))
        want = (loss(*up) - loss(*down)) / (2 * step)
        terms = grad.double().cpu() * d
        # the difference's third-order term is below step^2 of the terms' size, its cancellation below 1e-16 / step; the gradient
        # has some ten binary32 roundings of terms that are up to a few times itself
        assert abs(float(terms.sum()) - want) <= (100 * U + 100 * step ** 2 + 1e-9) * float(terms.abs().sum() + 1.0)


# ---- 4-bit weights --------------------------------------------------------------------------------------------------

def unpacked(codes, cols):
    b = codes.cpu().numpy().astype(np.int64)
    q = np.stack(((b & 15 ^ 8) - 8, (b >> 4 ^ 8) - 8), -1).reshape(b.shape[0], -1)
    return torch.from_numpy(q)


def per_column(scales, cols, group):
    return scales.double().cpu()[:, torch.arange(cols) // group]


COLS = [1, 2, 31, 32, 33, 64, 100, 128, 129, 255, 1000, 4096, 4999]


@gpu
@pytest.mark.parametrize("scale", ["f32", "bf16"])
@pytest.mark.parametrize("name", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("cols", COLS)
def test_group_quantize_and_dequantize(cols, group, name, scale):
    t, st, rows = TYPES[name], TYPES[scale], 13
    g = torch.Generator().manual_seed(cols * 10 + group)
    w = randn(g, rows, cols, std=0.02, t=t)
    w[3] = 0.0
    w[5] = (torch.randint(-15, 16, (cols,), generator=g) / 2.0).to(t)  # ties: halves of the step where the largest is 7
    w[5, ::group] = 7.0
    G = -(-cols // group)
    codes, scales, out = Guarded((rows, gq.w4_row_bytes(cols)), torch.uint8), Guarded((rows, G), st), Guarded((rows, cols), t)
    gq.group_quantize(w.to(DEV), group, codes.t, scales.t)
    gq.group_dequantize(codes.t, scales.t, group, out.t)
    assert codes.intact() and scales.intact() and out.intact()
    padded = torch.nn.functional.pad(w, (0, G * group - cols)).reshape(rows, G, group)
    want = (padded.float().abs().amax(2) * torch.tensor(1.0 / 7.0)).to(st)     # one product in binary32 and one rounding: the same bits
    assert torch.equal(scales.t.cpu(), want)
    s = per_column(want, cols, group)
    quotient = torch.where(s > 0, w.double() / s, 0.0)                # 24-bit numbers: nearest and ties come out right in 64 bits
    q = unpacked(codes.t, cols)
    assert torch.equal(q[:, :cols], quotient.round().clamp(-7, 7).long()) and not q[:, cols:].any()
    value = q[:, :cols].double() * s
    close(out.t, value, (U + half_step(t)) * value.abs() + least(t))


@gpu
@pytest.mark.parametrize("scale", ["f32", "bf16"])
def test_group_quantize_of_what_cannot_be_scaled(scale):
    st = TYPES[scale]
    w = torch.randn(6, 128)
    w[0, 3], w[1, 40], w[2, 127] = float("nan"), float("inf"), float("-inf")
    w[3] = 1e-45
    w[4] *= 1e38 / w[4].abs().max()
    codes, scales = torch.empty(6, 64, dtype=torch.uint8, device=DEV), torch.empty(6, 4, dtype=st, device=DEV)
    gq.group_quantize(w.to(DEV), 32, codes, scales)
    s, q = scales.float().cpu(), unpacked(codes, 128).reshape(6, 4, 32)
    bad = torch.zeros(6, 4, dtype=torch.bool)
    bad[0, 0] = bad[1, 1] = bad[2, 3] = True
    assert torch.equal(torch.isnan(s), bad) and not q[bad].any()
    assert not s[3].any() and not q[3].any()
    fine = ~bad
    fine[3] = False
    want = (w.reshape(6, 4, 32).double() / s.double()[:, :, None]).round().clamp(-7, 7).long()
    assert torch.equal(q[fine], want[fine]) and int(q[fine].abs().amax(1).min()) == 7
    out = torch.empty(6, 128, device=DEV)
    gq.group_dequantize(codes, scales, 32, out)
    assert torch.equal(torch.isnan(out.cpu().reshape(6, 4, 32)).all(2), bad) and not out[3].any()


def weights(g, rows, cols, group, st, low=-8):
    """Random codes (with -8 among them: a nibble that gq_group_quantize never writes) and scales, as tensors on the GPU."""
    q = torch.zeros(rows, 2 * gq.w4_row_bytes(cols), dtype=torch.int64)
    q[:, :cols] = torch.randint(low, 8, (rows, cols), generator=g)
    codes = ((q[:, 0::2] & 15) | ((q[:, 1::2] & 15) << 4)).to(torch.uint8)
    scales = (0.01 + torch.rand(rows, -(-cols // group), generator=g)).to(st)
    return q[:, :cols], codes.to(DEV), scales.to(DEV)


def plain_matvec(x, xs, q, scales, group, bias):
    """(y in 64 bits, its tolerance before the output's rounding)."""
    rows, cols = q.shape
    x, G = x.double(), -(-cols // group)
    s = scales.double().cpu()
    pad = G * group - cols
    xg = torch.nn.functional.pad(x, (0, pad)).reshape(x.shape[0], G, group)
    qg = torch.nn.functional.pad(q.double(), (0, pad)).reshape(rows, G, group)
    part = torch.einsum("mgk,rgk->mrg", xg, qg) * s[None]
    y = part.sum(2)
    tol = (G + 3) * U * part.abs().sum(2)                             # the product with the scale, the sum over groups, x_scales
    if xs is None:
        # a group's sum of (24 + code) x, at most 32 |x| a term, and the correction: at most group + 2 roundings of up to the
        # sum of the terms' sizes
        tol = tol + (group + 4) * U * torch.einsum("mgk,rg->mr", 32 * xg.abs(), s.abs())
    else:
        y, tol = y * xs.double()[:, None], tol * xs.double()[:, None].abs()
    if bias is not None:
        y = y + bias.double()
        tol = tol + U * (y.abs() + tol)
    return y, tol


MATVEC = [(1, 1, 1), (1, 3, 31), (2, 16, 32), (1, 17, 33), (5, 64, 127), (1, 100, 128), (16, 33, 129), (17, 48, 1000), (3, 255, 4096),
          (33, 40, 513), (64, 129, 640), (65, 31, 200), (130, 16, 96), (1, 1000, 2500), (8, 5, 9000)]


@gpu
@pytest.mark.parametrize("x_type,out,scale", [("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"), ("f16", "f16", "f32"), ("f16", "f32", "bf16"),
                                             ("i8", "bf16", "f32"), ("i8", "f32", "bf16"), ("i8", "f16", "f32")])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,rows,cols", MATVEC)
def test_w4_matvec(m, rows, cols, group, x_type, out, scale):
    g = torch.Generator().manual_seed(m * 7919 + rows * 31 + cols + group)
    q, codes, scales = weights(g, rows, cols, group, TYPES[scale])
    if x_type == "i8":
        x, xs = torch.randint(-128, 128, (m, cols), generator=g).to(torch.int8), 0.01 + torch.rand(m, generator=g)
    else:
        x, xs = randn(g, m, cols, t=TYPES[x_type]), None
    t = TYPES[out]
    for bias in (None, randn(g, rows, std=5.0, t=t)):
        y = Guarded((m, rows), t)
        gq.w4_matvec(x.to(DEV), codes, scales, group, y.t, x_scales=None if xs is None else xs.to(DEV), bias=None if bias is None else bias.to(DEV))
        want, tol = plain_matvec(x, xs, q, scales, group, bias)
        if t == torch.float16:
            want[want.abs() > 65519.0] *= float("inf")
        close(y.t, want, tol + half_step(t) * (want.abs() + tol) + least(t))
        assert y.intact()
    again = torch.empty_like(y.t)
    gq.w4_matvec(x.to(DEV), codes, scales, group, again, x_scales=None if xs is None else xs.to(DEV), bias=bias.to(DEV))
    assert torch.equal(again, y.t)                                    # no result depends on scheduling


@gpu
@pytest.mark.parametrize("x_type", ["bf16", "f16"])
def test_w4_matvec_rows_are_apart(x_type):
    """A row of x that is not finite gives NaN and leaves the others alone; so does a row of weights with a scale of NaN."""
    g = torch.Generator().manual_seed(5)
    q, codes, scales = weights(g, 50, 300, 32, torch.float32)
    x = randn(g, 20, 300, t=TYPES[x_type])
    clean = torch.empty(20, 50, device=DEV)
    gq.w4_matvec(x.to(DEV), codes, scales, 32, clean)
    x[3, 299], x[7, 0], x[18, 33] = float("nan"), float("inf"), float("-inf")
    scales[11, 4] = float("nan")
    y = torch.empty(20, 50, device=DEV)
    gq.w4_matvec(x.to(DEV), codes, scales, 32, y)
    bad = torch.zeros(20, 50, dtype=torch.bool, device=DEV)
    bad[3], bad[7], bad[18], bad[:, 11] = True, True, True, True
    assert torch.equal(torch.isnan(y), bad) and torch.equal(y[~bad], clean[~bad])


# every shape of workgroup that the rule chooses from: few and many rows of x, from a few rows of weights to over 16384
@gpu
@pytest.mark.parametrize("x_type,out,scale,group", [("bf16", "f32", "bf16", 128), ("f16", "f16", "f32", 64), ("i8", "f32", "bf16", 32)])
@pytest.mark.parametrize("m,rows,cols", [(1, 9001, 260), (2, 12000, 2100), (3, 9001, 260), (8, 17001, 136), (8, 40, 9001), (12, 5000, 1100), (12, 9001, 260),
                                         (12, 12000, 136), (12, 17001, 136), (30, 5000, 600), (30, 9001, 260), (30, 12000, 136), (30, 17001, 136),
                                         (50, 5000, 600), (50, 9001, 260), (50, 12000, 136), (50, 17001, 136), (100, 9001, 136),
                                         (40, 700, 4200), (12, 12000, 3200), (50, 12000, 1700), (30, 17001, 1700)])       # several steps
def test_w4_matvec_of_many_rows(m, rows, cols, group, x_type, out, scale):
    g = torch.Generator().manual_seed(m * 7919 + rows * 31 + cols + group)
    q, codes, scales = weights(g, rows, cols, group, TYPES[scale])
    if x_type == "i8":
        x, xs = torch.randint(-128, 128, (m, cols), generator=g).to(torch.int8), 0.01 + torch.rand(m, generator=g)
    else:
        x, xs = randn(g, m, cols, std=0.1, t=TYPES[x_type]), None
    t = TYPES[out]
    y = Guarded((m, rows), t)
    gq.w4_matvec(x.to(DEV), codes, scales, group, y.t, x_scales=None if xs is None else xs.to(DEV))
    want, tol = plain_matvec(x, xs, q, scales, group, None)
    close(y.t, want, tol + half_step(t) * (want.abs() + tol) + least(t))
    assert y.intact()


@gpu
def test_w4_matvec_without_columns_is_the_bias():
    codes, scales = torch.empty(5, 0, dtype=torch.uint8, device=DEV), torch.empty(5, 0, device=DEV)
    y, bias = torch.full((3, 5), 9.0, device=DEV), torch.arange(5.0, device=DEV)
    gq.w4_matvec(torch.empty(3, 0, dtype=torch.bfloat16, device=DEV), codes, scales, 32, y, bias=bias)
    assert torch.equal(y, bias.expand(3, 5))
    gq.w4_matvec(torch.empty(3, 0, dtype=torch.bfloat16, device=DEV), codes, scales, 32, y)
    assert not y.any()


@gpu
def test_codes_of_whole_rows_are_those_of_the_packed_format():
    """Where rows are a multiple of 32 long the codes are a GQ_PACK_I4 buffer: the integer sum of one worker unfolds them."""
    w = torch.randn(9, 256, device=DEV)
    codes, scales = torch.empty(9, 128, dtype=torch.uint8, device=DEV), torch.empty(9, 4, device=DEV)
    gq.group_quantize(w, 64, codes, scales)
    agg = torch.empty(9 * 256, dtype=torch.int32, device=DEV)
    gq.int_aggregate([codes], None, 9 * 256, gq.make_params(gq.GQ_LINEAR, 7, gq.GQ_PACK_I4), agg)
    assert torch.equal(agg.cpu().view(9, 256).long(), unpacked(codes, 256))


# ---- together -------------------------------------------------------------------------------------------------------

@gpu
def test_norm_in_front_of_a_projection():
    """As tokens are generated: the weights made into codes, the residual stream updated in place, the norm's int8 codes into the product."""
    g = torch.Generator().manual_seed(8)
    m, n, rows, group = 3, 1000, 200, 64
    w = randn(g, rows, n, std=0.05, t=torch.bfloat16)
    codes, scales = torch.empty(rows, gq.w4_row_bytes(n), dtype=torch.uint8, device=DEV), torch.empty(rows, -(-n // group), device=DEV)
    gq.group_quantize(w.to(DEV), group, codes, scales)
    x, res, nw = randn(g, m, n, t=torch.bfloat16), randn(g, m, n, std=2.0, t=torch.bfloat16), (1 + randn(g, n, std=0.1)).to(torch.bfloat16)
    stream = res.to(DEV)
    q, xs, y = torch.empty(m, n, dtype=torch.int8, device=DEV), torch.empty(m, device=DEV), torch.empty(m, rows, device=DEV)
    gq.rms_norm(x.to(DEV), nw.to(DEV), 1e-5, q, residual=stream, sum_out=stream, scales_out=xs)
    gq.w4_matvec(q, codes, scales, group, y, x_scales=xs)
    want, tol = plain_matvec(q.cpu(), xs.cpu(), unpacked(codes, n)[:, :n], scales, group, None)
    close(y, want, tol)
    h, _, _, _, yn, _ = plain_norm(x, res, nw, 1e-5, None)
    # half a code of every activation, half a code of every weight, and both
    dq = xs.double().cpu()[:, None] * 0.5001 + 0 * yn
    dw = per_column(scales, n, group) * 0.5001
    full = yn @ w.double().t()
    close(y, full, dq @ w.double().abs().t() + yn.abs() @ dw.t() + dq @ dw.t() + tol)


@gpu
def test_a_training_step_of_the_block():
    """Dropout of a branch and the norm in one call, its backward, and dropout alone: the same mask everywhere; the gradients then
    go through the exchange."""
    rows, n = 70, 515
    x, res, dy, ds = (torch.randn(rows, n, device=DEV) for _ in range(4))
    w = torch.ones(n, device=DEV)
    drop = gq.make_dropout(0.5, 4242, worker=6, index_base=1 << 33, rng_bits=16)
    h, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device=DEV)
    gq.rms_norm(x, w, 1e-6, y, residual=res, sum_out=h, rstd_out=rstd, drop=drop)
    alone = torch.empty_like(x)
    gq.dropout(x, drop, alone, res)
    assert torch.equal(alone, h)
    dx, dres, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(n, device=DEV)
    gq.rms_norm_backward(dy, h, w, rstd, dx, dsum=ds, dres_out=dres, dweight_out=dw, drop=drop)
    back = torch.empty_like(x)
    gq.dropout(dres, drop, back)
    assert torch.equal(back, dx)
    norm, agg, mean = torch.empty(1, device=DEV), torch.empty(n, dtype=torch.int32, device=DEV), torch.empty(n, device=DEV)
    gq.global_norm([dw, dw], gq.GQ_NORM_LINF, norm)
    gq.fused_quantize_aggregate([dw, dw], norm, gq.make_params(gq.GQ_LINEAR, 127, seed=1), 0, agg, mean)
    assert float((mean - dw).abs().max()) <= float(norm) / 127


@gpu
def test_on_another_stream_and_from_a_graph():
    rows, n, m, group = 40, 1030, 4, 32
    g = torch.Generator().manual_seed(3)
    x, res, dy = (randn(g, rows, n, t=torch.bfloat16).to(DEV) for _ in range(3))
    w = torch.ones(n, device=DEV, dtype=torch.bfloat16)
    wm = randn(g, 60, n, t=torch.bfloat16).to(DEV)
    drop = gq.make_dropout(0.2, 11)

    def buffers():
        e = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device=DEV)                # noqa: E731
        return {"drop": e(rows, n), "h": e(rows, n), "y": e(rows, n), "rstd": e(rows, t=torch.float32), "dx": e(rows, n), "dres": e(rows, n),
                "dw": e(n, t=torch.float32), "q": e(rows, n, t=torch.int8), "xs": e(rows, t=torch.float32),
                "codes": e(60, gq.w4_row_bytes(n), t=torch.uint8), "scales": e(60, -(-n // group)), "wm": e(60, n), "p": e(rows, 60),
                "p16": e(rows, 60, t=torch.float32)}

    def step(b, stream=None, workspace=None):
        gq.dropout(x, drop, b["drop"], res, stream=stream)
        gq.rms_norm(x, w, 1e-5, b["y"], residual=res, sum_out=b["h"], rstd_out=b["rstd"], drop=drop, stream=stream)
        ws = gq.rms_norm_backward(dy, b["h"], w, b["rstd"], b["dx"], dsum=res, dres_out=b["dres"], dweight_out=b["dw"], drop=drop,
                                  workspace=workspace, stream=stream)
        gq.rms_norm(b["y"], w, 1e-5, b["q"], scales_out=b["xs"], stream=stream)
        gq.group_quantize(wm, group, b["codes"], b["scales"], stream=stream)
        gq.group_dequantize(b["codes"], b["scales"], group, b["wm"], stream=stream)
        gq.w4_matvec(b["q"], b["codes"], b["scales"], group, b["p"], x_scales=b["xs"], stream=stream)
        gq.w4_matvec(b["y"], b["codes"], b["scales"], group, b["p16"], stream=stream)
        return ws
    same = lambda a, b: all(torch.equal(a[k], b[k]) for k in a)                              # noqa: E731
    want = buffers()
    step(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        got = buffers()
        side.wait_stream(torch.cuda.current_stream())
        step(got, stream)
        side.synchronize()
        assert same(got, want)
    # two graphs with a workspace each, replayed with eager work between
    graphs = []
    for _ in range(2):
        got, graph = buffers(), torch.cuda.CUDAGraph()
        ws = torch.empty(gq.rms_norm_workspace_bytes(rows, n), dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            step(got, workspace=ws)
        graphs.append((graph, got, ws))
    for _ in range(3):
        for graph, got, _ in graphs:
            for v in got.values():
                v.zero_()
        for graph, _, _ in graphs:
            graph.replay()
        eager = buffers()
        step(eager)
        torch.cuda.synchronize()
        assert same(eager, want) and all(same(got, want) for _, got, _ in graphs)


# ---- more than 2^32 elements or bytes: the last rows are those of a call on them alone ------------------------------

def filled(rows, n):
    return torch.empty(rows, n, dtype=torch.bfloat16, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(rows))


@gpu
@pytest.mark.parametrize("n", [65_536, 65_535])
def test_dropout_beyond_32_bits(n):
    rows, last = 66_000, 65_992
    x = filled(rows, n)
    out, tail = torch.empty_like(x), torch.empty_like(x[last:])
    gq.dropout(x, gq.make_dropout(0.3, 9), out)
    gq.dropout(x[last:], gq.make_dropout(0.3, 9, index_base=65_536 * last), tail)
    assert torch.equal(out[last:], tail) and 0.29 < float((tail == 0).float().mean()) < 0.31


@gpu
@pytest.mark.parametrize("n", [4096, 4095])
def test_rms_norm_beyond_32_bits(n):
    rows, last = 1_050_000, 1_049_992
    x, w = filled(rows, n), torch.ones(n, device=DEV)
    out, h = torch.empty_like(x), torch.empty_like(x)
    rstd, tail, th, tr = torch.empty(rows, device=DEV), torch.empty_like(x[last:]), torch.empty_like(x[last:]), torch.empty(8, device=DEV)
    drop, part = gq.make_dropout(0.3, 9, rng_bits=16), gq.make_dropout(0.3, 9, index_base=4096 * last, rng_bits=16)
    gq.rms_norm(x, w, 1e-5, out, sum_out=h, rstd_out=rstd, drop=drop)
    gq.rms_norm(x[last:], w, 1e-5, tail, sum_out=th, rstd_out=tr, drop=part)
    assert torch.equal(out[last:], tail) and torch.equal(h[last:], th) and torch.equal(rstd[last:], tr)
    gq.rms_norm_backward(x, h, w, rstd, out, drop=drop)
    gq.rms_norm_backward(x[last:], th, w, tr, tail, drop=part)
    assert torch.equal(out[last:], tail)


@gpu
@pytest.mark.parametrize("cols", [16_384, 16_380])
def test_weights_beyond_32_bits(cols):
    rows, last, group = 530_000, 529_992, 64
    w = filled(rows, cols)
    codes = torch.empty(rows, gq.w4_row_bytes(cols), dtype=torch.uint8, device=DEV)
    scales = torch.empty(rows, -(-cols // group), device=DEV)
    gq.group_quantize(w, group, codes, scales)
    tc, ts = torch.empty_like(codes[last:]), torch.empty_like(scales[last:])
    gq.group_quantize(w[last:], group, tc, ts)
    assert codes.numel() > 1 << 32 and torch.equal(codes[last:], tc) and torch.equal(scales[last:], ts)
    x = filled(9, cols)
    for m in (1, 9):
        y, t = torch.empty(m, rows, device=DEV), torch.empty(m, 8, device=DEV)
        gq.w4_matvec(x[:m], codes, scales, group, y)
        gq.w4_matvec(x[:m], tc, ts, group, t)
        want, tol = plain_matvec(x[:m].cpu(), None, unpacked(tc, cols)[:, :cols], ts, group, None)
        close(y[:, last:], want, tol)
        close(t, want, tol)
    gq.group_dequantize(codes, scales, group, w)
    t = torch.empty_like(w[last:])
    gq.group_dequantize(tc, ts, group, t)
    assert torch.equal(w[last:], t)
