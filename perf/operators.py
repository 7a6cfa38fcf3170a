"""The integer operators for activations without a calibrated grid, and the calls that are measured.

Three operators, each with one right value for every output:

* ``quantize``: rows of int16 or int32 values to int8 tokens, each row on a scale of its own;
* ``linear``: the int8 product of such tokens with int8 weights, with the token's scale, the
  output channel's multiplier and bias, and optionally a residual term in one rounding;
* ``groupnorm``: group normalization over an utterance's valid frames, channels last, with
  the integer Swish or without an activation.

The plain forms here are elementary torch operations in 64-bit integers; the sums of the
matrix product run in 32-bit floats over at most 1024 products each, where every partial sum
is a whole number of at most 2^24.
"""

from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

BITS = {"int8": 8, "int16": 16, "int32": 32}
DTYPE = {"int8": torch.int8, "int16": torch.int16, "int32": torch.int32}
LARGEST_LINEAR = 2.0 * 23000 * 4096 * 1024  # operations
LARGEST_QUANTIZE = 23000 * 4096             # elements
LARGEST_NORM = 48 * 1000 * 1024             # elements


def listed():
    return [
        # the Swish outputs of one 16-frame chunk of a live stream, nothing but latency
        {"name": "quantize_chunk", "op": "quantize", "rows": 16, "d": 1024, "type": "int16"},
        # int32 rows (wide sums) of 200 s of audio
        {"name": "quantize_wide", "op": "quantize", "rows": 2500, "d": 1024, "type": "int32"},
        # a feed-forward module's hidden activations on a full server batch
        {"name": "quantize_server", "op": "quantize", "rows": 23000, "d": 4096, "type": "int16"},
        # a single frame through one projection: reading the weights
        {"name": "linear_frame", "op": "linear", "rows": 1, "K": 1024, "N": 1024, "out": "int16", "residual": False},
        # one 10 s utterance through a feed-forward module's second layer, with the residual add
        {"name": "linear_10s", "op": "linear", "rows": 125, "K": 4096, "N": 1024, "out": "int8", "residual": True},
        # the scores of 1025 output tokens (an odd row length) for 200 s of audio
        {"name": "linear_head", "op": "linear", "rows": 2500, "K": 1024, "N": 1025, "out": "int32", "residual": False},
        # a feed-forward module's first layer on sixteen utterances of 30 s
        {"name": "linear_batch", "op": "linear", "rows": 6000, "K": 1024, "N": 4096, "out": "int16", "residual": False},
        # its second layer on a full server batch
        {"name": "linear_server", "op": "linear", "rows": 23000, "K": 4096, "N": 1024, "out": "int8", "residual": True},
        # one 10 s utterance between a convolution module's depthwise and second pointwise convolutions
        {"name": "groupnorm_10s", "op": "groupnorm", "B": 1, "T": 125, "low": 125, "d": 1024, "G": 32, "in": "int16",
         "out": "int16", "act": True},
        # the batched request, ragged lengths, to the next layer's static int8 grid
        {"name": "groupnorm_batch", "op": "groupnorm", "B": 16, "T": 375, "low": 200, "d": 1024, "G": 32,
         "in": "int16", "out": "int8", "act": True},
        # 200 s of audio in one piece on int8 grids, no activation
        {"name": "groupnorm_longform", "op": "groupnorm", "B": 1, "T": 2500, "low": 2500, "d": 1024, "G": 16,
         "in": "int8", "out": "int8", "act": False},
        # a full server batch
        {"name": "groupnorm_server", "op": "groupnorm", "B": 48, "T": 1000, "low": 500, "d": 1024, "G": 32,
         "in": "int16", "out": "int16", "act": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(("quantize", "linear", "linear", "groupnorm", "groupnorm"))
        if op == "quantize":
            case = {"op": op, "rows": _log_int(rng, 1, 23000), "d": 16 * _log_int(rng, 4, 256),
                    "type": rng.choice(("int16", "int16", "int32"))}
            if case["rows"] * case["d"] * BITS[case["type"]] <= LARGEST_QUANTIZE * 16:
                return case
        elif op == "linear":
            case = {"op": op, "rows": _log_int(rng, 1, 23000), "K": 16 * _log_int(rng, 4, 256),
                    "N": _log_int(rng, 4, 256) * 16 if rng.random() < 0.7 else _log_int(rng, 64, 4096),
                    "out": rng.choice(("int8", "int16", "int32"))}
            case["residual"] = case["out"] != "int32" and rng.random() < 0.5
            if work(case)["flops"] <= LARGEST_LINEAR:
                return case
        else:
            d = 64 * _log_int(rng, 4, 32)
            T = _log_int(rng, 1, 2500)
            case = {"op": op, "B": _log_int(rng, 1, 64), "T": T,
                    "low": T if rng.random() < 0.3 else max(1, int(T * rng.uniform(0.3, 1.0))), "d": d,
                    "G": rng.choice([g for g in (1, 2, 4, 8, 16, 32, 64) if d % g == 0]),
                    "in": rng.choice(("int8", "int16", "int16")), "out": rng.choice(("int8", "int16")),
                    "act": rng.random() < 0.7}
            if case["B"] * T * d <= LARGEST_NORM:
                return case


def work(case):
    """Each input read once, each output written once; padded frames are written (as zeros),
    not read.  Operations: 2 x the multiply-accumulates of the product; otherwise the few
    integer operations an element needs."""
    if case["op"] == "quantize":
        n = case["rows"] * case["d"]
        return {"bytes": n * (BITS[case["type"]] / 8 + 1.0) + 4.0 * case["rows"], "flops": 8.0 * n}
    if case["op"] == "linear":
        R, K, N = case["rows"], case["K"], case["N"]
        out = BITS[case["out"]] / 8.0
        return {"bytes": R * K + 4.0 * R + N * K + 12.0 * N + R * N * out * (2 if case["residual"] else 1),
                "flops": 2.0 * R * K * N}
    n = case["B"] * case["T"] * case["d"]
    valid = case["B"] * (case["low"] + case["T"]) / 2.0 * case["d"]
    return {"bytes": valid * BITS[case["in"]] / 8 + n * BITS[case["out"]] / 8.0 + 12.0 * case["d"],
            "flops": (25.0 if case["act"] else 12.0) * valid}


# ---------------------------------------------------------------------------------
# Inputs and integer constants, as an offline tool derives them from real-valued scales.

UNIT16 = 1.0 / 4096  # int16 grids of unit-variance activations (+-8)
UNIT8 = 1.0 / 32     # int8 grids (+-4)
GRID = {"int8": UNIT8, "int16": UNIT16}
SWISH_A, SWISH_C = -0.1240, 2.4632  # the polynomial's minimax pair


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape):
    return torch.randn(shape, generator=g, device="cuda")


def _uniform(g, shape, lo, hi):
    return lo + (hi - lo) * torch.rand(shape, generator=g, device="cuda")


def _clip(v, bits):
    lim = 2 ** (bits - 1) - 1
    return torch.round(v.double()).clamp(-lim, lim).to({8: torch.int8, 16: torch.int16, 32: torch.int32}[bits])


def _rows(g, rows, d, kind):
    """Activations whose spread differs from token to token and with heavy-tailed channels."""
    gain = torch.exp(0.7 * _normal(g, (rows, 1)))
    channel = torch.exp(0.5 * _normal(g, (1, d)))
    unit = 2.0 ** (BITS[kind] - 5)
    return _clip(_normal(g, (rows, d)) * gain * channel * (unit / 4.0), BITS[kind])


def _linear_constants(g, case):
    """mult, bias, shift and m_z for tokens of about 2^-5 of their range (rms) and weights of
    standard deviation 40: outputs of about unit variance on the output grid."""
    K, N, out = case["K"], case["N"], case["out"]
    p = 16 - (K - 1).bit_length()
    spread = 40.0 * 30.0 * math.sqrt(K) * 2.0 ** (p - 1 - 3)  # of t: the row's largest value about 2^-3 of the range
    unit = {"int8": 32.0, "int16": 4096.0, "int32": spread / 4}[out]
    shift = min(62, max(32, math.ceil(22 + math.log2(spread / unit))))
    mult = torch.round(_uniform(g, (N,), 0.5, 1.5).double() * (unit / spread * 2.0 ** shift)).to(torch.int32)
    bias = torch.round(_uniform(g, (N,), -0.5, 0.5).double() * unit * 2.0 ** (shift - 8)).to(torch.int64) * 256
    m_z = int(0.8 * 2.0 ** (shift - 16)) if case["residual"] else 0
    return mult, bias, shift, m_z


def _norm_constants(g, case):
    d, bits_in = case["d"], BITS[case["in"]]
    unit = 1.0 / GRID["int16" if case["act"] else case["out"]]
    # gn_mult = gamma unit 2^(shift - (bits_in - 1)), about 2^22
    shift = 22 - int(math.log2(unit)) + bits_in - 1
    mult = torch.round(_uniform(g, (d,), 0.5, 1.5).double() * unit * 2.0 ** (shift - bits_in + 1)).to(torch.int32)
    bias = torch.round(_uniform(g, (d,), -0.5, 0.5).double() * unit * 2.0 ** shift).to(torch.int64)
    eps = max(1, int(1e-5 / GRID[case["in"]] ** 2 * 65536))
    su = UNIT16 / 2
    sw_qc, sw_q1 = math.floor(SWISH_C / su), math.floor(1.0 / (SWISH_A * su * su))
    ratio = UNIT16 / (2.0 * -sw_q1) / GRID[case["out"]]
    shift_sw = 16 - math.floor(math.log2(ratio))
    return {"mult": mult, "bias": bias, "shift": shift, "eps": eps, "sw_qc": sw_qc, "sw_q1": sw_q1,
            "m_sw": int(round(ratio * 2.0 ** shift_sw)), "shift_sw": shift_sw}


def _inputs(case, seed):
    g = _gen(seed)
    if case["op"] == "quantize":
        return {"x": _rows(g, case["rows"], case["d"], case["type"])}
    if case["op"] == "linear":
        R, K, N = case["rows"], case["K"], case["N"]
        st = {"q": _clip(_normal(g, (R, K)) * _uniform(g, (R, 1), 20.0, 40.0), 8),
              "s": (torch.exp(0.7 * _normal(g, (R,)).double().clamp(-2.9, 2.9)) * 2.0 ** 28).to(torch.int32),
              "w": _clip(_normal(g, (N, K)) * 40.0, 8),
              "z": _clip(_normal(g, (R, N)) / GRID[case["out"]], BITS[case["out"]]) if case["residual"] else None}
        st["mult"], st["bias"], st["shift"], st["m_z"] = _linear_constants(g, case)
        return st
    B, T, d = case["B"], case["T"], case["d"]
    lengths = np.random.default_rng(seed).integers(case["low"], T + 1, size=B).astype(np.int32)
    lengths[seed % B] = T  # padded to the longest
    channel = torch.exp(0.5 * _normal(g, (1, 1, d)))
    z = (_normal(g, (B, T, d)) * channel + 0.3 * _normal(g, (1, 1, d))) * _uniform(g, (B, 1, 1), 0.4, 1.2)
    return {"z": _clip(z / GRID[case["in"]], BITS[case["in"]]), "lengths": lengths, **_norm_constants(g, case)}


def prepare(case, seed):
    st = {**_inputs(case, seed), "case": case}
    if own:
        from paper_2609_30846_amd import ipk

        st["ipk"] = ipk
        code = {"int8": ipk.IPK_INT8, "int16": ipk.IPK_INT16, "int32": ipk.IPK_INT32}
        if case["op"] == "linear":
            p = SimpleNamespace(w=st["w"].cpu().numpy(), mult=st["mult"].cpu().numpy(), bias=st["bias"].cpu().numpy(),
                                shift=st["shift"], m_z=st["m_z"], out_type=code[case["out"]])
            st["module"] = ipk.Linear(p)
        if case["op"] == "groupnorm":
            p = SimpleNamespace(d_model=case["d"], n_groups=case["G"], in_type=code[case["in"]],
                                out_type=code[case["out"]], gn_mult=st["mult"].cpu().numpy(),
                                gn_bias=st["bias"].cpu().numpy(), gn_shift=st["shift"], eps=st["eps"],
                                swish=case["act"], sw_qc=st["sw_qc"], sw_q1=st["sw_q1"], m_sw=st["m_sw"],
                                shift_sw=st["shift_sw"])
            st["module"] = ipk.GroupNorm(p, max_batch=case["B"], max_T=case["T"])
    return st


# ---------------------------------------------------------------------------------
# The plain forms


def run(st):
    case = st["case"]
    if own:
        if case["op"] == "quantize":
            return st["ipk"].quantize_tokens(st["x"])
        if case["op"] == "linear":
            return st["module"](st["q"], st["s"], z=st["z"])
        return st["module"](st["z"], lengths=st["lengths"])
    if case["op"] == "quantize":
        return _quantize(st["x"], BITS[case["type"]])
    if case["op"] == "linear":
        return _linear(st, case)
    return _groupnorm(st, case)


def _quantize(x, bits):
    x = x.to(torch.int64)
    alpha = x.abs().amax(1, keepdim=True).clamp(max=2 ** (bits - 1) - 1)
    q = torch.div(254 * x + alpha, 2 * alpha.clamp(min=1), rounding_mode="floor").clamp(-127, 127)
    return q.to(torch.int8), (alpha[:, 0] << (32 - bits)).to(torch.int32)


def _product(q, w):
    """q w^T as whole numbers: 32-bit float sums over at most 1024 products of at most 127^2."""
    R, K = q.shape
    N, c = w.shape[0], -(-K // 1024)
    pad = c * 1024 - K
    a = torch.nn.functional.pad(q.float(), (0, pad)).view(R, c, 1024).transpose(0, 1).contiguous()
    b = torch.nn.functional.pad(w.float(), (0, pad)).view(N, c, 1024).permute(1, 2, 0).contiguous()
    return torch.bmm(a, b).to(torch.int64).sum(0)


def _linear(st, case):
    p = 16 - (case["K"] - 1).bit_length()
    t = ((_product(st["q"], st["w"]) << p) * st["s"].to(torch.int64)[:, None]) >> 32
    v = t * st["mult"].to(torch.int64) + (st["bias"] + (1 << (st["shift"] - 1)))
    if st["z"] is not None:
        v = v + (st["z"].to(torch.int64) << 16) * st["m_z"]
    lim = 2 ** (BITS[case["out"]] - 1) - 1
    return (v >> st["shift"]).clamp(-lim, lim).to(DTYPE[case["out"]])


def _isqrt(v):
    r = torch.sqrt(v.double()).to(torch.int64)
    r = torch.where(r * r > v, r - 1, r)
    return torch.where((r + 1) * (r + 1) <= v, r + 1, r)


def _swish(h, st):
    a = h.abs()
    poly = (a.clamp(max=st["sw_qc"]) - st["sw_qc"]) ** 2 + st["sw_q1"]
    q = -(a * poly + h * st["sw_q1"])
    return (q * st["m_sw"] + (1 << (st["shift_sw"] - 1))) >> st["shift_sw"]


def _groupnorm(st, case):
    B, T, d, G = case["B"], case["T"], case["d"], case["G"]
    bits, lim = BITS[case["in"]], 2 ** (BITS[case["out"]] - 1) - 1
    lengths = torch.as_tensor(st["lengths"], device="cuda").to(torch.int64)
    valid = (torch.arange(T, device="cuda")[None, :] < lengths[:, None])[:, :, None]
    z = torch.where(valid, st["z"].to(torch.int64), 0)
    by_group = z.view(B, T, G, d // G)
    n = (lengths * (d // G))[:, None]
    S, Q = by_group.sum((1, 3)), (by_group * by_group).sum((1, 3))
    m0 = torch.div(S, n, rounding_mode="floor")
    r = S - n * m0
    D = Q - m0 * (2 * S - n * m0) - torch.div(r * r, n, rounding_mode="floor")
    whole = torch.div(D, n, rounding_mode="floor")
    V = (whole << 16) + torch.div((D - whole * n) << 16, n, rounding_mode="floor")
    R = torch.div(1 << 55, _isqrt((V + st["eps"]) << 16), rounding_mode="floor")
    mu = torch.div((S << 17) + n, 2 * n, rounding_mode="floor")
    R, mu = (v.repeat_interleave(d // G, 1) for v in (R, mu))
    gamma = st["mult"].to(torch.int64)
    # gamma R passes 64 bits: its floor by 2^24 from the two parts of R
    A = (gamma * (R >> 24) + ((gamma * (R & 0xFFFFFF)) >> 24)) >> (16 - bits)
    mean = (mu >> 16) * A + (((mu & 0xFFFF) * A) >> 16)
    C = st["bias"] + (1 << (st["shift"] - 1)) - mean
    h = (z * A[:, None, :] + C[:, None, :]) >> st["shift"]
    if case["act"]:
        h = _swish(h.clamp(-32767, 32767), st)
    return torch.where(valid, h.clamp(-lim, lim), 0).to(DTYPE[case["out"]])


# ---------------------------------------------------------------------------------
# The same values from the definitions, written apart: products in 64-bit floats (whole
# numbers far below 2^53), divisions instead of shifts, the statistics in Python's integers.


def _floordiv(a, b):
    return torch.div(a, b, rounding_mode="floor")


def exact(case, seed):
    st = _inputs(case, seed)
    if case["op"] == "quantize":
        x, lim = st["x"].to(torch.int64), 2 ** (BITS[case["type"]] - 1) - 1
        alpha = torch.maximum(x.max(1).values, -x.min(1).values).clamp(max=lim)
        num, den = 254 * x + alpha[:, None], 2 * alpha[:, None].clamp(min=1)
        q = (num - torch.remainder(num, den)) // den
        return q.clamp(-127, 127).to(torch.int8), (alpha * 2 ** (31 - lim.bit_length())).to(torch.int32)
    if case["op"] == "linear":
        K = case["K"]
        acc = (st["q"].double() @ st["w"].double().T.contiguous()).to(torch.int64)
        p = 16 - math.ceil(math.log2(K))
        t = _floordiv(acc * 2 ** p * st["s"].to(torch.int64)[:, None], 2 ** 32)
        v = t * st["mult"].to(torch.int64)[None] + st["bias"][None]
        if st["z"] is not None:
            v += st["z"].to(torch.int64) * (2 ** 16 * st["m_z"])
        y = _floordiv(v + 2 ** (st["shift"] - 1), 2 ** st["shift"])
        lim = torch.iinfo(DTYPE[case["out"]]).max
        return torch.minimum(torch.maximum(y, torch.tensor(-lim, device=y.device)),
                             torch.tensor(lim, device=y.device)).to(DTYPE[case["out"]])
    B, T, d, G = case["B"], case["T"], case["d"], case["G"]
    cg, bits = d // G, BITS[case["in"]]
    gamma, beta = st["mult"].tolist(), st["bias"].tolist()
    out = torch.zeros((B, T, d), dtype=torch.int64, device="cuda")
    for b in range(B):
        L = int(st["lengths"][b])
        z = st["z"][b, :L].to(torch.int64)
        sums, squares = z.sum(0).view(G, cg).sum(1).tolist(), z.square().sum(0).view(G, cg).sum(1).tolist()
        A, C = [], []
        for g in range(G):
            n, S, Q = L * cg, sums[g], squares[g]
            m0 = S // n
            D = Q - 2 * m0 * S + n * m0 * m0 - (S - n * m0) ** 2 // n
            R = 2 ** 55 // math.isqrt((D * 2 ** 16 // n + st["eps"]) * 2 ** 16)
            mu = (2 ** 17 * S + n) // (2 * n)
            for c in range(g * cg, (g + 1) * cg):
                A.append(gamma[c] * R // 2 ** (40 - bits))
                C.append(beta[c] - mu * A[-1] // 2 ** 16)
        A, C = (torch.tensor(v, dtype=torch.int64, device="cuda") for v in (A, C))
        out[b, :L] = _floordiv(z * A + C + 2 ** (st["shift"] - 1), 2 ** st["shift"])
        if case["act"]:
            h = out[b, :L].clamp(-32767, 32767)
            u = torch.minimum(h.abs(), torch.tensor(st["sw_qc"], device="cuda")) - st["sw_qc"]
            # -(|h| L + h q1) with L = u^2 + q1: -h (u^2 + 2 q1) for h >= 0, h u^2 below
            q = torch.where(h >= 0, -h * (u * u + 2 * st["sw_q1"]), h * (u * u))
            out[b, :L] = _floordiv(q * st["m_sw"] + 2 ** (st["shift_sw"] - 1), 2 ** st["shift_sw"])
    lim = torch.iinfo(DTYPE[case["out"]]).max
    return out.clamp(-lim, lim).to(DTYPE[case["out"]])
