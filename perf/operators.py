"""The calls that a user of this library makes for the layers around the gradient exchange, as cases that can be timed and compared:
dropout from the counter-based generator, root-mean-square norm with the residual's addition (forward with an output in the input's
type or in 8 bits, and backward), 4-bit weights under group scales (making and unfolding them) and their product with a few rows.

Kinds:

  dropout   gq.dropout: out = residual + dropout(x); a training step's backward is the same call on the gradient
  norm      gq.rms_norm: h = residual + dropout(x), y = h / rms(h) * weight, y in the input's type or in e4m3 under a scale per row
  backward  gq.rms_norm_backward: the gradients of x, of the residual and of the weight
  weights   gq.group_quantize -> gq.group_dequantize: weights to 4-bit codes under group scales, and the values that they stand for
  matvec    gq.w4_matvec: rows of activations (bf16, fp16, or int8 codes under a scale per row) times 4-bit weights, bias
  serve     gq.rms_norm (int8 codes out) -> gq.w4_matvec: what stands in front of a projection when tokens are generated

`own` false: the same results from elementary torch operations in 32 bits.  Random numbers are those of Philox4x32-10 (Salmon et al.,
SC'11) with counter (lo32(g / 4), hi32(g / 4), worker, 3) and key (lo32(seed), hi32(seed)), word g mod 4, for element (r, c) with
g = index_base + 8 ceil(n / 8) r + c; with 16 bits counter (lo32(g / 8), hi32(g / 8), worker, 3), half g mod 2 of word (g mod 8) / 2.
"""
import math

import torch

own = False

M32 = 0xFFFFFFFF
DOMAIN = 3
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "i8": 1, "e4m3": 1}


def _dropout(name, rows, n, dtype, p, bits, residual):
    return {"name": name, "kind": "dropout", "rows": rows, "n": n, "dtype": dtype, "p": p, "bits": bits, "residual": residual}


def _norm(name, rows, n, dtype, weight, out, residual, p, bits):
    return {"name": name, "kind": "norm", "rows": rows, "n": n, "dtype": dtype, "weight": weight, "out": out, "residual": residual,
            "p": p, "bits": bits}


def _backward(name, rows, n, dtype, weight, dsum, p, bits):
    return {"name": name, "kind": "backward", "rows": rows, "n": n, "dtype": dtype, "weight": weight, "dsum": dsum, "p": p,
            "bits": bits}


def _weights(name, rows, cols, dtype, group, scale):
    return {"name": name, "kind": "weights", "rows": rows, "cols": cols, "dtype": dtype, "group": group, "scale": scale}


def _matvec(name, m, rows, cols, x, group, scale, out, bias):
    return {"name": name, "kind": "matvec", "m": m, "rows": rows, "cols": cols, "x": x, "group": group, "scale": scale, "out": out,
            "bias": bias}


def _serve(name, m, rows, cols, dtype, group, scale):
    return {"name": name, "kind": "serve", "m": m, "rows": rows, "cols": cols, "dtype": dtype, "group": group, "scale": scale}


def listed():
    return [
        # one token through a square projection: latency
        _matvec("matvec_1_4096x4096_bf16", 1, 4096, 4096, "bf16", 128, "bf16", "bf16", False),
        # one token through a wide projection of a large model, activations in int8: the weights' bytes
        _matvec("matvec_1_28672x8192_i8", 1, 28672, 8192, "i8", 64, "f32", "bf16", False),
        # a batch of tokens, odd sizes, small groups, with a bias
        _matvec("matvec_61_14335x4095_f16", 61, 14335, 4095, "f16", 32, "bf16", "f16", True),
        # the norm in front of a projection and the projection, one token
        _serve("serve_1_12288x4096", 1, 12288, 4096, "bf16", 128, "bf16"),
        # a batch of tokens in front of an 8-bit product, odd row length
        _norm("norm_61x5003_e4m3", 61, 5003, "f16", "f16", "e4m3", True, 0.0, 32),
        # a training step's tokens: dropout of the branch, the residual stream, the norm of the next block
        _norm("norm_8192x4096_dropout", 8192, 4096, "bf16", "bf16", "same", True, 0.1, 32),
        # its backward
        _backward("backward_8192x4096_dropout", 8192, 4096, "bf16", "bf16", True, 0.1, 32),
        # the backward of a small odd model in full precision
        _backward("backward_1000x2047_f32", 1000, 2047, "f32", "f32", False, 0.0, 32),
        # one small odd vector: latency
        _dropout("dropout_100003_f32", 1, 100_003, "f32", 0.1, 32, False),
        # a long training batch's activations, short draws
        _dropout("dropout_16384x8192_bf16", 16384, 8192, "bf16", 0.2, 16, True),
        # one matrix of a large model, when its weights are made into codes
        _weights("weights_8192x8192_bf16", 8192, 8192, "bf16", 128, "bf16"),
        # a small odd matrix in full precision, small groups
        _weights("weights_1001x4999_f32", 1001, 4999, "f32", 32, "f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["dropout", "norm", "backward", "weights", "matvec", "matvec", "serve"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    p = rng.choice([0.0, 0.1, rng.uniform(0.01, 0.9)])
    bits = rng.choice([32, 16])
    if kind == "dropout":
        n = _log_int(rng, 100, 30000)
        case = _dropout("", _log_int(rng, 1, max(1, 60_000_000 // n)), n, dtype, max(p, 0.05), bits, rng.random() < 0.5)
    elif kind in ("norm", "backward"):
        n = _log_int(rng, 64, 16384)
        rows = _log_int(rng, 1, max(1, 30_000_000 // n))
        weight = rng.choice([dtype, "f32"])
        case = (_norm("", rows, n, dtype, weight, rng.choice(["same", "same", "e4m3"]), rng.random() < 0.7, p, bits) if kind == "norm"
                else _backward("", rows, n, dtype, weight, rng.random() < 0.5, p, bits))
    else:
        rows, cols = _log_int(rng, 64, 16384), _log_int(rng, 64, 14000)
        group, scale = rng.choice([32, 64, 128]), rng.choice(["f32", "bf16"])
        m = _log_int(rng, 1, 64)
        if kind == "weights":
            case = _weights("", rows, min(cols, 60_000_000 // rows), dtype, group, scale)
        elif kind == "matvec":
            x = rng.choice(["bf16", "f16", "i8"])
            out = rng.choice(["f32", "bf16"]) if x == "i8" else rng.choice([x, x, "f32"])
            case = _matvec("", m, rows, cols, x, group, scale, out, rng.random() < 0.3)
        else:
            case = _serve("", m, rows, cols, dtype if dtype != "f32" else "bf16", group, scale)
    return {k: v for k, v in case.items() if k != "name"}


def _row_bytes(cols):
    return (cols + 31) // 32 * 16


def _groups(case):
    return -(-case["cols"] // case["group"])


def work(case):
    k = case["kind"]
    if k in ("dropout", "norm", "backward"):
        e, size = case["rows"] * case["n"], SIZE[case["dtype"]]
        if k == "dropout":
            return {"bytes": e * size * (3 if case["residual"] else 2), "flops": 2 * e}
        wsize = case["n"] * SIZE[case["weight"]]
        if k == "norm":
            out = size if case["out"] == "same" else 1
            apart = case["residual"] or case["p"] > 0                 # the sum is an output of its own
            return {"bytes": e * (size + out + size * (bool(case["residual"]) + apart)) + 4 * case["rows"] + wsize, "flops": 5 * e}
        return {"bytes": e * size * (3 + bool(case["dsum"]) + (case["p"] > 0)) + 4 * case["rows"] + wsize + 4 * case["n"], "flops": 9 * e}
    codes = case["rows"] * _row_bytes(case["cols"]) + case["rows"] * _groups(case) * SIZE[case["scale"]]
    if k == "weights":
        return {"bytes": 2 * case["rows"] * case["cols"] * SIZE[case["dtype"]] + 2 * codes, "flops": 3 * case["rows"] * case["cols"]}
    m = case["m"]
    flops = 2 * m * case["rows"] * case["cols"]
    if k == "matvec":
        return {"bytes": codes + m * case["cols"] * SIZE[case["x"]] + m * case["rows"] * SIZE[case["out"]], "flops": flops}
    return {"bytes": codes + m * case["cols"] * SIZE[case["dtype"]] * 3 + m * case["rows"] * SIZE[case["dtype"]], "flops": flops}


# ---- inputs -------------------------------------------------------------------------------------------------------

def _randn(g, *shape, std=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g)


def _tokens(g, rows, n, std):
    """Activations: normal, a few channels much larger than the others, as in trained models."""
    x = _randn(g, rows, n, std=std)
    return x.mul_(torch.where(torch.rand(n, generator=g, device="cuda") < 0.004, 20.0, 1.0))


def _codes(g, rows, cols):
    """Weights as codes -7 .. 7, two to a byte (the even column in the low half), rows of whole 16 bytes, zeros behind the last column."""
    q = torch.zeros(rows, 2 * _row_bytes(cols), dtype=torch.int8, device="cuda")
    q[:, :cols] = _randn(g, rows, cols, std=2.3).round_().clamp_(-7, 7)
    return ((q[:, 0::2] & 15) | (q[:, 1::2] << 4)).view(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1_000_003 + 17)
    s, k = {"case": case, "seed": (seed * 0x9E3779B97F4A7C15 + 12345) & ((1 << 64) - 1)}, case["kind"]
    if k in ("dropout", "norm", "backward"):
        rows, n, t = case["rows"], case["n"], TYPES[case["dtype"]]
        s["worker"], s["base"] = 3, 8 * (seed % 1000) + (1 << 33)      # a later layer's offset in the step's stream
        new = lambda dt=t: torch.empty(rows, n, dtype=dt, device="cuda")  # noqa: E731
        if k == "dropout":
            s["x"], s["out"] = _tokens(g, rows, n, 1.0).to(t), new()
            s["residual"] = _tokens(g, rows, n, 3.0).to(t) if case["residual"] else None
            return s
        s["w"] = (1.0 + _randn(g, n, std=0.2)).to(TYPES[case["weight"]])
        if k == "norm":
            s["x"] = _tokens(g, rows, n, 1.0).to(t)
            s["residual"] = _tokens(g, rows, n, 3.0).to(t) if case["residual"] else None
            s["sum"] = new() if case["residual"] or case["p"] > 0 else None
            s["out"] = new(t if case["out"] == "same" else torch.float8_e4m3fn)
            s["scales"] = None if case["out"] == "same" else torch.empty(rows, device="cuda")
            s["rstd"] = torch.empty(rows, device="cuda")
            return s
        s["h"] = _tokens(g, rows, n, 3.0).to(t)
        s["rstd"] = (s["h"].double().square().mean(1) + EPS).rsqrt().float()
        s["dy"] = _randn(g, rows, n, std=1e-2).to(t)
        s["dsum"] = _randn(g, rows, n, std=1e-2).to(t) if case["dsum"] else None
        s["dres"], s["dx"] = (new() if case["p"] > 0 else None), new()
        s["dw"] = torch.empty(n, device="cuda")
        return s
    rows, cols = case["rows"], case["cols"]
    st = TYPES[case["scale"]]
    if k == "weights":
        s["w"] = _tokens(g, rows, cols, 0.02).to(TYPES[case["dtype"]])
        s["codes"] = torch.empty(rows, _row_bytes(cols), dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty(rows, _groups(case), dtype=st, device="cuda")
        s["values"] = torch.empty_like(s["w"])
        return s
    m = case["m"]
    s["codes"] = _codes(g, rows, cols)
    s["scales"] = (0.004 + 0.008 * torch.rand(rows, _groups(case), generator=g, device="cuda")).to(st)
    if k == "matvec":
        s["bias"] = _randn(g, rows).to(TYPES[case["out"]]) if case["bias"] else None
        s["out"] = torch.empty(m, rows, dtype=TYPES[case["out"]], device="cuda")
        if case["x"] == "i8":
            s["x"] = _randn(g, m, cols, std=30.0).round_().clamp_(-127, 127).to(torch.int8)
            s["xs"] = 0.01 + 0.02 * torch.rand(m, generator=g, device="cuda")
        else:
            s["x"], s["xs"] = _tokens(g, m, cols, 1.0).to(TYPES[case["x"]]), None
        return s
    t = TYPES[case["dtype"]]
    s["x"], s["residual"] = _tokens(g, m, cols, 1.0).to(t), _tokens(g, m, cols, 3.0).to(t)
    s["w"] = (1.0 + _randn(g, cols, std=0.2)).to(t)
    s["sum"], s["q"] = torch.empty_like(s["x"]), torch.empty(m, cols, dtype=torch.int8, device="cuda")
    s["xs"], s["out"] = torch.empty(m, device="cuda"), torch.empty(m, rows, dtype=t, device="cuda")
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------

def _high(a, c):
    """The upper 32 bits of the product of the 32-bit number a and 32-bit numbers c held in 64 bits."""
    return (a * (c >> 16) + ((a * (c & 0xFFFF)) >> 16)) >> 16


def _philox(call, worker, seed):
    """The four random words of each call, one row of four a call."""
    c0, c1 = call & M32, call >> 32
    c2, c3 = torch.full_like(call, worker), torch.full_like(call, DOMAIN)
    k0, k1 = seed & M32, seed >> 32
    for _ in range(10):
        h0, l0 = _high(0xD2511F53, c0), (0xD2511F53 * c0) & M32
        h1, l1 = _high(0xCD9E8D57, c2), (0xCD9E8D57 * c2) & M32
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return torch.stack((c0, c1, c2, c3), 1)


def _threshold(p, bits):
    return min(round(p * (1 << bits)), (1 << bits) - 1)


def _dropped(x32, s):
    """x32 with what the generator drops set to zero and the rest scaled to keep the mean."""
    case = s["case"]
    rows, n, bits = case["rows"], case["n"], case["bits"]
    t = _threshold(case["p"], bits)
    if t == 0:
        return x32
    pitch, per = -(-n // 8) * 8, 4 if bits == 32 else 8
    words = _philox(s["base"] // per + torch.arange(rows * pitch // per, device="cuda"), s["worker"], s["seed"])
    if bits == 16:
        words = torch.stack((words & 0xFFFF, words >> 16), 2)
    kept = words.reshape(rows, pitch)[:, :n] >= t
    return torch.where(kept, x32 * torch.tensor((1 << bits) / ((1 << bits) - t), dtype=torch.float32, device="cuda"), 0.0)


def _rms(h, w):
    """(y, 1 / rms) of rows of h; the long sum in 64 bits."""
    rstd = (1.0 / (h.double().square().mean(1, keepdim=True) + EPS).sqrt()).float()
    return (h * rstd) * w.float(), rstd


def _unfold(codes, scales, cols, group):
    q = torch.stack(((codes << 4).view(torch.int8) >> 4, codes.view(torch.int8) >> 4), 2).reshape(codes.shape[0], -1)[:, :cols]
    return q.float() * scales.float().repeat_interleave(group, 1)[:, :cols]


def _plain(s):
    case = s["case"]
    k = case["kind"]
    if k == "dropout":
        y = _dropped(s["x"].float(), s)
        return {"out": (y if s["residual"] is None else s["residual"].float() + y).to(s["x"].dtype)}
    if k == "norm":
        h = _dropped(s["x"].float(), s)
        h = h if s["residual"] is None else s["residual"].float() + h
        y, rstd = _rms(h, s["w"])
        out = {"rstd": rstd[:, 0]}
        if s["sum"] is not None:
            out["sum"] = h.to(s["x"].dtype)
        if case["out"] == "same":
            return out | {"out": y.to(s["x"].dtype)}
        scale = y.abs().amax(1, keepdim=True) / 448.0
        return out | {"out": (y * (1.0 / scale)).to(torch.float8_e4m3fn), "scales": scale[:, 0]}
    if k == "backward":
        dy, xh = s["dy"].float(), s["h"].float() * s["rstd"][:, None]
        g = dy * s["w"].float()
        dh = (g - xh * (g.double() * xh).mean(1, keepdim=True).float()) * s["rstd"][:, None]
        dh = dh if s["dsum"] is None else s["dsum"].float() + dh
        dw = (dy.double() * xh).sum(0).float()
        if case["p"] > 0:
            return {"dres": dh.to(s["h"].dtype), "dx": _dropped(dh, s).to(s["h"].dtype), "dw": dw}
        return {"dx": dh.to(s["h"].dtype), "dw": dw}
    cols, group = case["cols"], case["group"]
    if k == "weights":
        w = torch.nn.functional.pad(s["w"].float(), (0, _groups(case) * group - cols)).reshape(case["rows"], -1, group)
        scale = (w.abs().amax(2) / 7.0).to(s["scales"].dtype)
        q = (w.double() / scale.double()[:, :, None]).round().clamp(-7, 7).float()       # next to a border 32 bits are too few
        values = q * scale.float()[:, :, None]
        return {"values": values.reshape(case["rows"], -1)[:, :cols].to(s["w"].dtype), "scales": scale}
    w = _unfold(s["codes"], s["scales"], cols, group)
    if k == "matvec":
        y = s["x"].float() @ w.t()
        y = y if s["xs"] is None else y * s["xs"][:, None]
        return {"out": (y if s["bias"] is None else y + s["bias"].float()).to(s["out"].dtype)}
    h = s["residual"].float() + s["x"].float()
    y, _ = _rms(h, s["w"])
    scale = y.abs().amax(1, keepdim=True) / 127.0
    q = (y * (1.0 / scale)).round().clamp(-127, 127)
    return {"sum": h.to(s["x"].dtype), "out": ((q @ w.t()) * scale).to(s["x"].dtype)}


# ---- the framework's calls ----------------------------------------------------------------------------------------

def _framework(s):
    import paper_2305_18627_amd as gq
    case = s["case"]
    k = case["kind"]
    if k in ("dropout", "norm", "backward"):
        drop = gq.make_dropout(case["p"], s["seed"], s["worker"], s["base"], case["bits"]) if case["p"] > 0 else None
    if k == "dropout":
        gq.dropout(s["x"], drop, s["out"], s["residual"])
        return {"out": s["out"]}
    if k == "norm":
        gq.rms_norm(s["x"], s["w"], EPS, s["out"], residual=s["residual"], sum_out=s["sum"], scales_out=s["scales"],
                    rstd_out=s["rstd"], drop=drop)
        return {key: s[key] for key in ("out", "rstd", "sum", "scales") if s[key] is not None}
    if k == "backward":
        gq.rms_norm_backward(s["dy"], s["h"], s["w"], s["rstd"], s["dx"], dsum=s["dsum"], dres_out=s["dres"], dweight_out=s["dw"],
                             drop=drop)
        return {key: s[key] for key in ("dres", "dx", "dw") if s[key] is not None}
    if k == "weights":
        gq.group_quantize(s["w"], case["group"], s["codes"], s["scales"])
        gq.group_dequantize(s["codes"], s["scales"], case["group"], s["values"])
        return {"values": s["values"], "scales": s["scales"]}
    if k == "matvec":
        gq.w4_matvec(s["x"], s["codes"], s["scales"], case["group"], s["out"], x_scales=s["xs"], bias=s["bias"])
        return {"out": s["out"]}
    gq.rms_norm(s["x"], s["w"], EPS, s["q"], residual=s["residual"], sum_out=s["sum"], scales_out=s["xs"])
    gq.w4_matvec(s["q"], s["codes"], s["scales"], case["group"], s["out"], x_scales=s["xs"])
    return {"sum": s["sum"], "out": s["out"]}


def run(state):
    return _framework(state) if own else _plain(state)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_kept(s, case):
    """Which elements are kept, and by what they are scaled: the generator in numpy's unsigned integers."""
    import numpy as np
    rows, n, bits = case["rows"], case["n"], case["bits"]
    pitch = (n + 7) & ~7
    first, count = (s["base"] // 4, rows * pitch // 4) if bits == 32 else (s["base"] // 8, rows * pitch // 8)
    call = np.arange(first, first + count, dtype=np.uint64)
    low = np.uint64(M32)
    ctr = [call & low, call >> np.uint64(32), np.uint64(s["worker"]), np.uint64(DOMAIN)]
    key = [s["seed"] & M32, s["seed"] >> 32]
    for r in range(10):
        p, q = np.uint64(0xD2511F53) * ctr[0], np.uint64(0xCD9E8D57) * ctr[2]
        a = np.uint64((key[0] + r * 0x9E3779B9) & M32)
        b = np.uint64((key[1] + r * 0xBB67AE85) & M32)
        ctr = [(q >> np.uint64(32)) ^ ctr[1] ^ a, q & low, (p >> np.uint64(32)) ^ ctr[3] ^ b, p & low]
    words = np.empty((count, 4), dtype=np.uint32)
    for j in range(4):
        words[:, j] = ctr[j]
    draws = words if bits == 32 else words.view(np.uint16)             # little-endian: the low half first
    t = _threshold(case["p"], bits)
    kept = draws.reshape(rows, pitch)[:, :n] >= t
    return torch.from_numpy(kept).cuda(), float(1 << bits) / float((1 << bits) - t)


def _exact_e4m3(v):
    """v on the grid of e4m3 (3 bits behind the leading one, smallest exponent -6), ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))).clamp_min(-6) - 3)
    return (torch.round(v / step) * step).clamp(-448.0, 448.0)


def _exact_weights(s, case):
    """The 4-bit weights' values, a row of columns at a time from the two halves of each byte."""
    b = s["codes"].to(torch.int64)
    q = torch.empty(b.shape[0], 2 * b.shape[1], dtype=torch.float64, device="cuda")
    q[:, 0::2], q[:, 1::2] = (((b & 15) ^ 8) - 8).double(), (((b >> 4) ^ 8) - 8).double()
    at = torch.arange(case["cols"], device="cuda") // case["group"]
    return q[:, :case["cols"]] * s["scales"].double()[:, at]


def exact(case, seed):
    s = prepare(case, seed)
    k = case["kind"]
    if k in ("dropout", "norm", "backward") and case["p"] > 0:
        kept, by = _exact_kept(s, case)
        drop = lambda v: torch.where(kept, v * by, torch.zeros_like(v))  # noqa: E731
    else:
        drop = lambda v: v  # noqa: E731
    if k == "dropout":
        y = drop(s["x"].double())
        return {"out": y if s["residual"] is None else y + s["residual"].double()}
    if k == "norm" or k == "serve":
        h = drop(s["x"].double())
        if s["residual"] is not None:
            h = h + s["residual"].double()
        rstd = 1.0 / torch.sqrt((h * h).sum(1) / h.shape[1] + EPS)
        y = h * rstd[:, None] * s["w"].double()
        top = y.abs().max(1).values
        if k == "serve":
            q = torch.round(y * (127.0 / top)[:, None])
            return {"sum": h, "out": q @ _exact_weights(s, case).t() * (top / 127.0)[:, None]}
        out = {"rstd": rstd} if s["sum"] is None else {"rstd": rstd, "sum": h}
        if case["out"] == "same":
            out["out"] = y
        else:
            out["out"], out["scales"] = _exact_e4m3(y * (448.0 / top)[:, None]), top / 448.0
        return out
    if k == "backward":
        rstd, h, dy = s["rstd"].double()[:, None], s["h"].double(), s["dy"].double()
        g = dy * s["w"].double()
        dh = rstd * g - h * rstd ** 3 * ((g * h).sum(1, keepdim=True) / h.shape[1])
        if s["dsum"] is not None:
            dh = dh + s["dsum"].double()
        dw = (dy * h * rstd).sum(0)
        return {"dres": dh, "dx": drop(dh), "dw": dw} if case["p"] > 0 else {"dx": dh, "dw": dw}
    if k == "weights":
        w, cols, group = s["w"].double(), case["cols"], case["group"]
        values, scales = torch.empty_like(w), []
        for c in range(0, cols, group):
            part = w[:, c:c + group]
            scale = (part.abs().max(1).values / 7.0).to(s["scales"].dtype).double()    # the scale is held in its own type
            values[:, c:c + group] = torch.round(part / scale[:, None]).clamp(-7, 7) * scale[:, None]
            scales.append(scale)
        return {"values": values, "scales": torch.stack(scales, 1)}
    y = s["x"].double() @ _exact_weights(s, case).t()
    if s["xs"] is not None:
        y = y * s["xs"].double()[:, None]
    return {"out": y if s["bias"] is None else y + s["bias"].double()}
