"""Microscaled 4-bit linear layers: the work that a training or serving program has them do, in the plain form and
through the framework's entry points.

The format: 32 consecutive values of a row (or of a column, for the products that contract over rows) share a
power-of-two scale 2^s held in 8 bits; each value is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, times 2^s.

Kinds of pass
  roundtrip  quantize a bf16 matrix along its rows, its columns or both and read it back: what a stored context
             stands for when the backward pass takes it up
  linear     Y = Q(X) W^T for bf16 activations and a weight that the program keeps quantized
  backward   dY with stochastic rounding, dX = dY W and dW = dY^T X on operands kept from the forward pass
  step       one training step of a layer whose weight the optimizer has just changed: W, X, Y, dY, dX, dW

A case's sizes: M tokens (rows), K input features, N output features (roundtrip: M rows, K columns).
"""
import math

import numpy as np
import torch

own = False

GROUP = 32
OUT = {"bf16": torch.bfloat16, "f32": torch.float32}

# The largest listed product, in multiply-adds, and the largest listed matrix of a round trip.
MAX_MACS = 8192 ** 3
MAX_ELEMENTS = 4096 * 11008


def listed():
    return [
        # one token of a decode step through an up projection: the weight's bytes are the work
        {"name": "linear_token", "kind": "linear", "M": 1, "K": 4096, "N": 11008, "out": "bf16"},
        # a handful of sequences decoding together through a down projection
        {"name": "linear_few_tokens", "kind": "linear", "M": 33, "K": 11008, "N": 4096, "out": "bf16"},
        # the smallest layer of the benchmark: launches and latency are all there is
        {"name": "linear_small", "kind": "linear", "M": 256, "K": 512, "N": 512, "out": "f32"},
        # a ragged batch through a layer whose sizes are no multiples of anything
        {"name": "linear_ragged", "kind": "linear", "M": 777, "K": 1544, "N": 2201, "out": "bf16"},
        # a full batch through an up projection
        {"name": "linear_up", "kind": "linear", "M": 4096, "K": 4096, "N": 11008, "out": "bf16"},
        # the square problem
        {"name": "linear_square", "kind": "linear", "M": 8192, "K": 8192, "N": 8192, "out": "bf16"},
        # backward of a full batch through a down projection
        {"name": "backward_down", "kind": "backward", "M": 4096, "K": 11008, "N": 4096, "out": "bf16"},
        # backward of a short ragged batch: a contraction over few tokens
        {"name": "backward_ragged", "kind": "backward", "M": 131, "K": 1544, "N": 2200, "out": "f32"},
        # a whole training step of a small layer
        {"name": "step_2048", "kind": "step", "M": 2048, "K": 2048, "N": 2048, "out": "bf16"},
        # a batch's activations stored along both axes, as a training step takes them
        {"name": "roundtrip_both", "kind": "roundtrip", "M": 4096, "K": 11008, "sides": "both", "rounding": "floor"},
        # a gradient with stochastic rounding
        {"name": "roundtrip_sr", "kind": "roundtrip", "M": 4096, "K": 4096, "sides": "both", "rounding": "stochastic"},
        # odd sizes, one side, scales that cover every value
        {"name": "roundtrip_odd", "kind": "roundtrip", "M": 1023, "K": 1001, "sides": "columns", "rounding": "cover"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _features(rng, lo, hi):
    """A feature dimension: mostly a multiple of 128, sometimes of 8 only, sometimes odd."""
    n, kind = _log_int(rng, lo, hi), rng.random()
    if kind < 0.6:
        return max(128, n // 128 * 128)
    return max(8, n // 8 * 8) if kind < 0.85 else n | 1


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "backward", "step", "roundtrip", "roundtrip"])
    if kind == "roundtrip":
        while True:
            case = {"kind": kind, "M": _log_int(rng, 1, 8192), "K": _features(rng, 64, 11008),
                    "sides": rng.choice(["rows", "columns", "both"]),
                    "rounding": rng.choice(["floor", "cover", "stochastic"])}
            if case["M"] * case["K"] <= MAX_ELEMENTS:
                return case
    products = {"linear": 1, "backward": 2, "step": 3}[kind]
    while True:
        M = _log_int(rng, 1 if kind == "linear" else 64, 8192)
        K, N = _features(rng, 64, 11008), _features(rng, 64, 11008)
        if products * M * K * N <= 0.8 * MAX_MACS:
            return {"kind": kind, "M": M, "K": K, "N": N, "out": rng.choice(["bf16", "bf16", "f32"])}


# ---- inputs ---------------------------------------------------------------------------------------


def _activation(g, M, K):
    """N(0, 1) with a few channels some 30 times as large, as activations in front of a projection have them."""
    x = torch.randn((M, K), device="cuda", generator=g)
    n = max(1, K // 500)
    x[:, torch.randperm(K, device="cuda", generator=g)[:n]] *= 30.0
    return x.to(torch.bfloat16)


def _weight(g, N, K):
    return (0.02 * torch.randn((N, K), device="cuda", generator=g)).to(torch.bfloat16)


def _gradient(g, M, N):
    """Heavy-tailed, with rows of padding tokens that are zero."""
    d = torch.randn((M, N), device="cuda", generator=g)
    d *= 1e-3 * torch.exp(torch.randn((M, N), device="cuda", generator=g))
    d[torch.rand((M,), device="cuda", generator=g) < 0.05] = 0.0
    return d.to(torch.bfloat16)


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    kind, M, K = case["kind"], case["M"], case["K"]
    if kind == "roundtrip":
        make = _gradient if case["rounding"] == "stochastic" else _activation
        return {"x": make(g, M, K)}
    t = {"x": _activation(g, M, K), "w": _weight(g, case["N"], K)}
    if kind != "linear":
        t["dy"] = _gradient(g, M, case["N"])
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    st = {"kind": case["kind"], "seed": int(seed), "case": case}
    if own:
        import paper_2503_08040_amd as fq
        st["fq"] = fq
    if case["kind"] == "roundtrip":
        st["x"] = t["x"]
        if own:
            sides = {"rows": fq.FQ_MX_ROWS, "columns": fq.FQ_MX_COLS, "both": fq.FQ_MX_BOTH}[case["sides"]]
            st["q"] = fq.MxTensor(case["M"], case["K"], sides)
        return st
    st["out"] = OUT[case["out"]]
    M, K, N = case["M"], case["K"], case["N"]
    if case["kind"] == "linear":
        st["x"] = t["x"]
        # the weight as a serving program keeps it
        if own:
            st["w"] = fq.fq_mx_quantize(t["w"])
            st["qx"] = fq.MxTensor(M, K, fq.FQ_MX_ROWS)
        else:
            st["w"] = _store(t["w"])
        return st
    st["dy"] = t["dy"]
    if case["kind"] == "backward":
        # kept from the forward pass: W and X along their columns
        if own:
            st["w"] = fq.fq_mx_quantize(t["w"], sides=fq.FQ_MX_COLS)
            st["x"] = fq.fq_mx_quantize(t["x"], sides=fq.FQ_MX_COLS)
            st["qdy"] = fq.MxTensor(M, N, fq.FQ_MX_BOTH)
        else:
            st["w"], st["x"] = _store(t["w"].T), _store(t["x"].T)
        return st
    st["x"], st["w"] = t["x"], t["w"]
    if own:
        for name, (rows, cols) in {"qw": (N, K), "qx": (M, K), "qdy": (M, N)}.items():
            st[name] = fq.MxTensor(rows, cols, fq.FQ_MX_BOTH)
    return st


# ---- the plain form -------------------------------------------------------------------------------


def _random16(rows, cols, seed):
    """16 random bits per element: Philox4x32-10 with key seed and counter (column / 8, row, 0, 0); element c of a row
    takes half c % 2 (the low half first) of word (c / 2) % 4."""
    mask = 0xFFFFFFFF
    blocks = -(-cols // 8)
    c0 = torch.arange(blocks, device="cuda").expand(rows, blocks)
    c1 = torch.arange(rows, device="cuda")[:, None].expand(rows, blocks)
    c2 = c3 = torch.zeros((1, 1), dtype=torch.int64, device="cuda").expand(rows, blocks)
    k0, k1 = seed & mask, (seed >> 32) & mask

    def product(a, b):
        # the high and the low half of a 32 x 32 bit product, in 64 bits with a sign
        low, high = a * (b & 0xFFFF), a * (b >> 16)
        mid = (low >> 16) + (high & 0xFFFF)
        return (high >> 16) + (mid >> 16), ((mid & 0xFFFF) << 16) | (low & 0xFFFF)

    for _ in range(10):
        h0, l0 = product(c0, 0xD2511F53)
        h1, l1 = product(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    words = torch.stack([c0, c1, c2, c3], dim=-1)
    halves = torch.stack([words & 0xFFFF, words >> 16], dim=-1)
    return halves.reshape(rows, blocks * 8)[:, :cols]


def _grouped(x, fill=0):
    """[rows, cols] -> [rows, groups, 32], padded with zeros."""
    rows, cols = x.shape
    return torch.nn.functional.pad(x, (0, -cols % GROUP), value=fill).view(rows, -1, GROUP)


def _power(s):
    """2^s for whole numbers s, from the bits of binary32."""
    return ((s.int() + 127) << 23).view(torch.float32)


def _codes(x, rounding, random=None):
    """(magnitude in half units with its sign, exponent of the scale) of the groups along the rows of a matrix."""
    v = _grouped(x.float())
    mant, exp = torch.frexp(v.abs().amax(dim=2, keepdim=True))
    s = exp - 3
    if rounding != "floor":
        s = s + (mant > 0.75)
    s = torch.where(mant == 0, torch.full_like(s, -127), s.clamp(min=-127))
    # |x| / 2^s in two factors, either of which binary32 has
    half = torch.div(s, 2, rounding_mode="floor")
    t = v.abs() * _power(-half) * _power(half - s)
    if rounding == "stochastic":
        fixed = (t * 2.0 ** 17).long()
        shift = (fixed >= 1 << 18).long() + (fixed >= 1 << 19).long()
        half_units = ((fixed + (_grouped(random) << shift)) >> (16 + shift)) << shift
    else:
        step = torch.where(t < 2, 0.5, torch.where(t < 4, 1.0, 2.0))
        half_units = 2.0 * (torch.round(t / step) * step).clamp(max=6.0)
    return torch.copysign(half_units.float(), v), s


def _values(q, s, cols):
    """What the codes stand for, binary32."""
    s = s.int()
    half = torch.div(s, 2, rounding_mode="floor")
    v = 0.5 * q.float() * _power(half) * _power(s - half)
    return v.flatten(1)[:, :cols]


def _plain(x, rounding="floor", random=None):
    return _values(*_codes(x, rounding, random), x.shape[1])


def _store(w):
    """A matrix as a program keeps it: 8 bits a value, 8 bits a scale, and its number of columns."""
    q, s = _codes(w, "floor")
    return q.to(torch.int8), s.to(torch.int8), w.shape[1]


def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_plain(st):
    kind = st["kind"]
    if kind == "roundtrip":
        x, case = st["x"], st["case"]
        stochastic = case["rounding"] == "stochastic"
        random = _random16(*x.shape, st["seed"]) if stochastic else None
        out = []
        if case["sides"] != "columns":
            out.append(_plain(x, case["rounding"], random).to(torch.bfloat16))
        if case["sides"] != "rows":
            out.append(_plain(x.T, case["rounding"], random.T if stochastic else None).T.to(torch.bfloat16))
        return out
    if kind == "linear":
        return (_plain(st["x"]) @ _values(*st["w"]).T).to(st["out"])
    dy = st["dy"]
    random = _random16(*dy.shape, st["seed"])
    dy_rows, dy_cols = _plain(dy, "stochastic", random), _plain(dy.T, "stochastic", random.T)
    if kind == "backward":
        w_cols, x_cols = _values(*st["w"]), _values(*st["x"])
        return (dy_rows @ w_cols.T).to(st["out"]), dy_cols @ x_cols.T
    y = (_plain(st["x"]) @ _plain(st["w"]).T).to(st["out"])
    dx = (dy_rows @ _plain(st["w"].T).T).to(st["out"])
    return y, dx, dy_cols @ _plain(st["x"].T).T


# ---- the framework's calls ------------------------------------------------------------------------


def _run_own(st):
    fq, kind = st["fq"], st["kind"]
    if kind == "roundtrip":
        case, q = st["case"], st["q"]
        if case["rounding"] == "stochastic":
            fq.fq_mx_quantize_sr(st["x"], st["seed"], out=q)
        else:
            rule = fq.FQ_MX_FLOOR if case["rounding"] == "floor" else fq.FQ_MX_COVER
            fq.fq_mx_quantize(st["x"], out=q, rule=rule)
        out = []
        if case["sides"] != "columns":
            out.append(fq.fq_mx_dequantize(q, fq.FQ_MX_ROWS))
        if case["sides"] != "rows":
            out.append(fq.fq_mx_dequantize(q, fq.FQ_MX_COLS))
        return out
    if kind == "linear":
        return fq.fq_mx_linear(st["x"], st["w"], xq=st["qx"], out_dtype=st["out"])
    if kind == "step":
        fq.fq_mx_quantize(st["w"], out=st["qw"])
        fq.fq_mx_quantize(st["x"], out=st["qx"])
        y = fq.fq_mx_gemm(fq.FQ_OP_NT, st["qx"], st["qw"], out_dtype=st["out"])
        w, x = st["qw"], st["qx"]
    else:
        w, x = st["w"], st["x"]
    fq.fq_mx_quantize_sr(st["dy"], st["seed"], out=st["qdy"])
    dx = fq.fq_mx_gemm(fq.FQ_OP_NN, st["qdy"], w, out_dtype=st["out"])
    dw = fq.fq_mx_gemm(fq.FQ_OP_TN, st["qdy"], x, out_dtype=torch.float32)
    return (y, dx, dw) if kind == "step" else (dx, dw)


# ---- what a pass cannot do without ----------------------------------------------------------------


def work(case):
    """Each call reads its inputs and writes its outputs once; 17 / 32 byte per quantized value and side."""
    kind, M, K = case["kind"], case["M"], case["K"]
    stored = 17.0 / 32.0
    if kind == "roundtrip":
        sides = 2 if case["sides"] == "both" else 1
        return {"bytes": int(M * K * (2 + sides * (2 * stored + 2))), "flops": 4 * sides * M * K}
    N, o = case["N"], 2 if case["out"] == "bf16" else 4
    macs = M * N * K
    if kind == "linear":
        return {"bytes": int(2 * M * K + stored * N * K + o * M * N), "flops": 2 * macs}
    # dY, its two sides written and read; W and X along their columns; dX and dW
    back = 2 * M * N + 4 * stored * M * N + stored * (N * K + M * K) + o * M * K + 4 * N * K
    if kind == "backward":
        return {"bytes": int(back), "flops": 4 * macs}
    # W and X, both sides written, the rows' read; Y
    fore = (2 + 3 * stored) * (N * K + M * K) + o * M * N
    return {"bytes": int(back + fore), "flops": 6 * macs}


# ---- the definition in 64 bits --------------------------------------------------------------------


def _exact_random16(rows, cols, seed):
    """The same generator on the host, in unsigned 64-bit words."""
    u32 = np.uint64(0xFFFFFFFF)
    blocks = (cols + 7) // 8
    ctr = np.zeros((4, rows, blocks), dtype=np.uint64)
    ctr[0] = np.arange(blocks, dtype=np.uint64)
    ctr[1] = np.arange(rows, dtype=np.uint64)[:, None]
    key = [seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32]
    for r in range(10):
        p0, p1 = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        k0, k1 = np.uint64((key[0] + r * 0x9E3779B9) % 2 ** 32), np.uint64((key[1] + r * 0xBB67AE85) % 2 ** 32)
        ctr = np.stack([(p1 >> np.uint64(32)) ^ ctr[1] ^ k0, p1 & u32, (p0 >> np.uint64(32)) ^ ctr[3] ^ k1, p0 & u32])
    out = np.empty((rows, blocks, 8), dtype=np.int32)
    for w in range(4):
        out[:, :, 2 * w] = ctr[w] & np.uint64(0xFFFF)
        out[:, :, 2 * w + 1] = ctr[w] >> np.uint64(16)
    return torch.from_numpy(out.reshape(rows, -1)[:, :cols].copy()).cuda()


def _exact_values(x, rounding="floor", random=None):
    """The values a bf16 matrix is quantized to along its rows, from the list of E2M1 values."""
    rows, cols = x.shape
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    out = torch.empty((rows, cols), dtype=torch.float64, device=x.device)
    chunk = max(GROUP, (1 << 24) // max(rows, 1) // GROUP * GROUP)
    for c in range(0, cols, chunk):
        v = x[:, c:c + chunk].double()
        n = v.shape[1]
        v = torch.nn.functional.pad(v, (0, -n % GROUP)).reshape(rows, -1, GROUP)
        top = v.abs().amax(dim=2, keepdim=True)
        # the exponents from the bits of binary64, in which no bf16 value is subnormal
        e = (top.clamp(min=2.0 ** -140).view(torch.int64) >> 52) - 1023
        s = e - 2
        if rounding != "floor":
            s = s + (top > 1.5 * ((e + 1023) << 52).view(torch.float64)).long()
        scale = ((s.clamp(min=-127) + 1023) << 52).view(torch.float64)
        t = v.abs() / scale
        below = (torch.bucketize(t, grid, right=True) - 1).clamp(max=7)      # the largest value of the list <= t
        above = (below + 1).clamp(max=7)
        lo, hi = grid[below], grid[above]
        gap = torch.where(hi > lo, hi - lo, torch.ones_like(lo))
        if rounding == "stochastic":
            r = torch.nn.functional.pad(random[:, c:c + chunk], (0, -n % GROUP)).reshape(rows, -1, GROUP).double()
            # up if the fraction of the step, in 2^-16 below a multiple of 2^-17 in t, and u reach a whole step
            frac = (torch.floor(t * 2.0 ** 17) / 2.0 ** 17 - lo) / gap
            up = frac * 65536.0 + r >= 65536.0
        else:
            frac = (t - lo) / gap
            up = (frac > 0.5) | ((frac == 0.5) & (below % 2 == 1))
        q = torch.where(up & (below < 7), hi, lo)
        out[:, c:c + n] = (torch.where(v < 0, -q, q) * scale).reshape(rows, -1)[:, :n]
    return out


def exact(case, seed):
    t = _inputs(case, seed)
    kind, x = case["kind"], t["x"]
    if kind == "roundtrip":
        how = case["rounding"]
        random = _exact_random16(*x.shape, int(seed)) if how == "stochastic" else None
        out = []
        if case["sides"] != "columns":
            out.append(_exact_values(x, how, random))
        if case["sides"] != "rows":
            out.append(_exact_values(x.T.contiguous(), how, None if random is None else random.T.contiguous()).T)
        return out
    w = t["w"]
    if kind == "linear":
        return _exact_values(x) @ _exact_values(w).T
    dy = t["dy"]
    random = _exact_random16(*dy.shape, int(seed))
    dx = _exact_values(dy, "stochastic", random) @ _exact_values(w.T.contiguous()).T
    dw = _exact_values(dy.T.contiguous(), "stochastic", random.T.contiguous()) @ _exact_values(x.T.contiguous()).T
    if kind == "backward":
        return dx, dw
    return _exact_values(x) @ _exact_values(w).T, dx, dw
