"""Performance cases of the operators that run an AFNO block's channel MLP in eight bits, one call through a
public entry point per case, with the operators' plain forms.

Operators ("op" of a case, "backward" its direction):
  pack        a tensor's rows in eight bits, and the values that they then stand for: an activation kept for the
              backward pass and read again.
  rms_norm    out = v / sqrt(mean(v^2) + eps) gamma of v = x + residual, in the storage type, in eight bits or
              both, and the sum v; the gradients dx and dgamma.
  linear      out = drop(act(x w + b)) + residual for rows and weights in eight bits, out in the storage type, in
              eight bits or both, and x w + b in eight bits; the gradients dx, dw, db of drop(act(x w + b)) from
              x and x w + b kept in eight bits.
Eight bits: the values v / 2^s rounded to E4M3 (four exponent bits, three of mantissa, largest 448), one
exponent s for every 32 neighbouring channels of a row, the smallest with which none of them is above 448, in
-117 .. 119; a row's last block is filled up with zeros.
drop() keeps element e (its flat index) where a 16-bit number of the counter-based generator Philox4x32
with seven rounds is at least T = 65536 p rounded, and scales by 65536 / (65536 - T).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
BLOCK = 32


def _pack(name, M, C, dtype):
    return {"name": name, "op": "pack", "backward": False, "M": M, "C": C, "dtype": dtype}


def _norm(name, M, C, dtype, residual=False, out=True, packed=False):
    return {"name": name, "op": "rms_norm", "backward": False, "M": M, "C": C, "dtype": dtype, "residual": residual,
            "out": out, "packed": packed}


def _norm_backward(name, M, C, dtype, residual=False):
    return {"name": name, "op": "rms_norm", "backward": True, "M": M, "C": C, "dtype": dtype, "residual": residual}


def _linear(name, M, K, N, dtype, act="gelu", p=0.0, residual=False, bias=True, out=True, packed=False, pre=False):
    return {"name": name, "op": "linear", "backward": False, "M": M, "K": K, "N": N, "dtype": dtype, "act": act, "p": p,
            "residual": residual, "bias": bias, "out": out, "packed": packed, "pre": pre}


def _linear_backward(name, M, K, N, dtype, act="gelu", p=0.0, bias=True):
    return {"name": name, "op": "linear", "backward": True, "M": M, "K": K, "N": N, "dtype": dtype, "act": act, "p": p,
            "bias": bias}


def listed():
    return [
        # the hidden layer's input on the 180 x 360 grid, kept for the backward pass in half the memory and read again
        _pack("pack_180x360_bf16", 64800, 1024, "bf16"),
        # an odd number of channels at full precision, on a regional grid
        _pack("pack_odd_fp32", 5187, 333, "fp32"),
        # the norm of one token on its way into an eight-bit product: a probe of one grid point, where latency counts
        _norm("rms_norm_1_token_bf16", 1, 1024, "bf16", residual=True, out=False, packed=True),
        # the sum of the residual stream and the filter's output, and its norm in eight bits
        _norm("rms_norm_180x360_bf16", 64800, 1024, "bf16", residual=True, out=False, packed=True),
        # the gradient through that norm, onto the gradient of the residual stream
        _norm_backward("rms_norm_backward_180x360_bf16", 64800, 1024, "bf16", residual=True),
        # an odd number of channels at full precision
        _norm_backward("rms_norm_backward_odd_fp32", 5187, 333, "fp32"),
        # one token through the MLP's first product, where latency and the weights count
        _linear("linear_1_token_bf16", 1, 1024, 4096, "bf16"),
        # the MLP's first product in training, 4,096 hidden units for 1,024 channels: what the next product and the
        # backward pass read, in eight bits
        _linear("linear_up_180x360_bf16", 64800, 1024, 4096, "bf16", p=0.1, out=False, packed=True, pre=True),
        # its second product, back to the channels and onto the residual stream
        _linear("linear_down_180x360_bf16", 64800, 4096, 1024, "bf16", act="none", p=0.1, residual=True),
        # a projection of sizes that no tile divides, with its result at full precision
        _linear("linear_ragged_fp32", 4095, 333, 77, "fp32", act="relu"),
        # the gradient of the first product from what was kept in eight bits
        _linear_backward("linear_backward_180x360_bf16", 64800, 1024, 4096, "bf16", p=0.1),
        # the same at full precision on a 2.5-degree grid
        _linear_backward("linear_backward_72x144_fp32", 10368, 384, 1536, "fp32"),
    ]


def _log(rng, low, high):
    return round(math.exp(rng.uniform(math.log(low), math.log(high))))


def _width(rng, low, high):
    """A width over the logarithm of the range: half of them multiples of 64, a fourth of 8, the rest of none."""
    n, u = _log(rng, low, high), rng.random()
    step = 64 if u < 0.5 and n >= 64 else 8 if u < 0.75 and n >= 8 else 1
    return max(1, n // step * step)


def draw(rng):
    """A case of the ranges above: one token to the 180 x 360 grid's 64,800, widths of 8 to 4,096."""
    while True:
        op = rng.choices(["linear", "rms_norm", "pack"], [6, 3, 1])[0]
        dtype = "bf16" if rng.random() < 0.65 else "fp32"
        backward, residual = rng.random() < 0.4, rng.random() < 0.5
        M = _log(rng, 1, 64800)
        packed = rng.random() < 0.6
        out = not packed or rng.random() < 0.3
        if op == "linear":
            K, N = _width(rng, 8, 4096), _width(rng, 8, 4096)
            p = 0.0 if rng.random() < 0.5 else round(rng.uniform(0.02, 0.6), 3)
            act = rng.choice(["none", "relu", "gelu", "gelu"])
            bias = rng.random() < 0.85
            # no dearer than the largest case listed, which is in bf16 and has 1.1e12 operations
            if (4.0 if backward else 2.0) * M * K * N > (1.0e12 if dtype == "bf16" or not backward else 3.0e11):
                continue
            if backward:
                c = _linear_backward("", M, K, N, dtype, act, p, bias)
            else:
                c = _linear("", M, K, N, dtype, act, p, residual, bias, out, packed, act != "none" and rng.random() < 0.4)
        else:
            C = _width(rng, 8, 4096)
            if M * C > 64800 * 1024:
                continue
            if op == "pack":
                c = _pack("", M, C, dtype)
            elif backward:
                c = _norm_backward("", M, C, dtype, residual)
            else:
                c = _norm("", M, C, dtype, residual, out, packed)
        del c["name"]
        return c


# ---------------------------------------------------------------- eight bits in elementary operations


def _blocks(v):
    """v [..., C] with zeros up to a whole block, as [..., blocks, 32]."""
    pad = -v.shape[-1] % BLOCK
    if pad:
        v = torch.nn.functional.pad(v, (0, pad))
    return v.reshape(*v.shape[:-1], -1, BLOCK)


def _power(e):
    """2^e as float32 for whole e in -126 .. 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _to_eight(v):
    """float32 rows in eight bits: E4M3 values [..., 32 blocks] and the exponents [..., blocks]."""
    b = _blocks(v)
    size = torch.where(torch.isfinite(b), b.abs(), 0.0).amax(-1)
    part, e = torch.frexp(size)  # size = part 2^e, part in 1/2 .. 1
    s = torch.where(size > 0, e - 9 + (part > 0.875), -117).clamp(-117, 119)
    q = torch.where(torch.isfinite(b), (b * _power(-s)[..., None]).clamp(-448.0, 448.0), math.nan)
    return q.to(torch.float8_e4m3fn).flatten(-2), s


def _from_eight(q, s, C):
    """The values that they stand for, in float32."""
    v = q.float().reshape(*s.shape, BLOCK) * _power(s)[..., None]
    return v.flatten(-2)[..., :C]


def _kept(v):
    """float32 rows as a program keeps them: E4M3 values, and an exponent byte s + 127 to a block."""
    q, s = _to_eight(v)
    return q.contiguous(), (s + 127).to(torch.uint8).view(torch.float8_e8m0fnu).contiguous()


def _kept_values(t, C):
    return _from_eight(t[0], t[1].view(torch.uint8).to(torch.int32) - 127, C)


# ---------------------------------------------------------------- inputs


def prepare(case, seed):
    c, dt, dev = case, DTYPES[case["dtype"]], torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(1000003 * int(seed) + 31)

    def normal(*shape, std=1.0, mean=0.0):
        return (mean + std * torch.randn(*shape, generator=g, device=dev)).to(dt)

    def uneven(*shape):
        """Activations whose channels differ in scale."""
        return torch.randn(*shape, generator=g, device=dev) * (0.5 + 1.5 * torch.rand(shape[-1], generator=g, device=dev))

    s = {"case": dict(c)}
    if c.get("p"):
        # the run's seed, this operator's place in the model, and the training step on the device
        s["seed"], s["offset"] = 0x9E3779B97F4A7C15 * (int(seed) + 1) % 2 ** 64, 3 << 40
        s["counter"] = torch.tensor([1000 + int(seed) % 1000], dtype=torch.int64, device=dev)
    if c["op"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        x, w = uneven(M, K), torch.randn(K, N, generator=g, device=dev) / math.sqrt(K)
        s["x"] = _kept(x)
        s["b"] = normal(N, std=0.1) if c["bias"] else None
        if c["backward"]:
            s["w"], s["g"] = w.to(dt), normal(M, N)
            if c["act"] != "none":
                z = x @ w
                s["pre"] = _kept(z + s["b"].float() if c["bias"] else z)
        else:
            s["w"] = _kept(w.t().contiguous())  # rows of K, as x
            if c["residual"]:
                s["residual"] = normal(M, N)
    else:
        M, C = c["M"], c["C"]
        s["x"] = (0.2 + uneven(M, C)).to(dt)
        if c["op"] == "rms_norm":
            s["gamma"] = normal(C, std=0.1, mean=1.0)
            if c["residual"]:
                s["residual"] = normal(M, C)
            if c["backward"]:
                s["g"] = normal(M, C)
    return s


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2208_05419_amd as afno
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    if c["op"] == "pack":
        return {"values": afno.mx8_unpack(afno.mx8_pack(s["x"]))}
    if c["op"] == "rms_norm":
        if c["backward"]:
            return afno.rms_norm_backward(s["g"], s["x"], s["gamma"], eps=EPS, gsum=s.get("residual"))
        v = torch.empty_like(s["x"]) if c["residual"] else None
        out = torch.empty_like(s["x"]) if c["out"] else None
        out8 = afno.mx8_empty(s["x"].shape, s["x"].device) if c["packed"] else None
        afno.rms_norm_forward(s["x"], s["gamma"], eps=EPS, residual=s.get("residual"), out=out, sum_out=v, out8=out8)
        d = {"sum": v, "out": out, "values": afno.mx8_unpack(out8) if c["packed"] else None}
        return {k: t for k, t in d.items() if t is not None}
    M, K, N = c["M"], c["K"], c["N"]
    rng = {"p": c["p"], "seed": s["seed"], "offset": s["offset"], "counter": s["counter"]} if c["p"] else {}
    x = afno.Mx8(*s["x"], K)
    if c["backward"]:
        pre = afno.Mx8(*s["pre"], N) if c["act"] != "none" else None
        d = afno.mx8_linear_backward(s["g"], x, s["w"], pre8=pre, activation=c["act"], bias=c["bias"], **rng)
        return {k: t for k, t in d.items() if t is not None}
    dev = s["x"][0].device
    out = torch.empty(M, N, dtype=dt, device=dev) if c["out"] else None
    out8 = afno.mx8_empty((M, N), dev) if c["packed"] else None
    pre8 = afno.mx8_empty((M, N), dev) if c["pre"] else None
    afno.mx8_linear_forward(x, afno.Mx8(*s["w"], K), s["b"], activation=c["act"], residual=s.get("residual"), dtype=dt,
                            out=out, out8=out8, pre8=pre8, **rng)
    d = {"out": out, "values": afno.mx8_unpack(out8) if c["packed"] else None, "pre": afno.mx8_unpack(pre8) if c["pre"] else None}
    return {k: t for k, t in d.items() if t is not None}


# ---------------------------------------------------------------- plain forms, in float32


def _threshold(p):
    return int(np.rint(float(np.float32(p)) * 65536.0))


def _keep(s, n):
    """Which of n elements the generator keeps."""
    low = 0xFFFFFFFF
    group = torch.arange((n + 7) // 8, dtype=torch.int64, device=s["counter"].device)
    place = s["counter"] + (s["offset"] - 2 ** 64 if s["offset"] >= 2 ** 63 else s["offset"])
    c0, c1, c2, c3 = group & low, group >> 32, place & low, (place >> 32) & low
    k0, k1 = s["seed"] & low, s["seed"] >> 32
    for _ in range(7):
        # the products' 64 bits wrap in a signed integer; their halves are right all the same
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], -1)
    return words.reshape(-1)[:n] >= _threshold(s["case"]["p"])


def _dropped(s, y):
    p = s["case"]["p"]
    if not p:
        return y
    return torch.where(_keep(s, y.numel()).reshape(y.shape), y * (65536.0 / (65536 - _threshold(p))), 0.0)


def _rounded(v):
    """float32 rows as the eight bits have them, in bfloat16, which holds every such value."""
    return _from_eight(*_to_eight(v), v.shape[-1]).to(torch.bfloat16)


def _run_plain(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    if c["op"] == "pack":
        return {"values": _rounded(s["x"].float())}
    if c["op"] == "rms_norm":
        x, d = s["x"].float(), {}
        if not c["backward"] and c["residual"]:
            d["sum"] = (x + s["residual"].float()).to(dt)
            x = d["sum"].float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        if not c["backward"]:
            y = x * r * s["gamma"].float()
            if c["out"]:
                d["out"] = y.to(dt)
            if c["packed"]:
                d["values"] = _rounded(y)
            return d
        h, g = x * r, s["g"].float()
        a = g * s["gamma"].float()
        dx = r * (a - h * (a * h).mean(-1, keepdim=True))
        if c["residual"]:
            dx = dx + s["residual"].float()
        return {"dx": dx.to(dt), "dgamma": (g * h).sum(0)}
    K, N = c["K"], c["N"]
    x = _kept_values(s["x"], K)
    if c["backward"]:
        dz = _dropped(s, s["g"].float())
        if c["act"] != "none":
            z = _kept_values(s["pre"], N)
            if c["act"] == "relu":
                dz = torch.where(z > 0, dz, 0.0)
            else:
                dz = dz * (0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi)))
        d = {"dx": (dz @ s["w"].float().t()).to(dt), "dw": (x.t() @ dz).to(dt)}
        return {**d, "db": dz.sum(0).to(dt)} if c["bias"] else d
    z = x @ _kept_values(s["w"], K).t()
    if c["bias"]:
        z = z + s["b"].float()
    y = torch.relu(z) if c["act"] == "relu" else 0.5 * z * torch.erfc(z * -math.sqrt(0.5)) if c["act"] == "gelu" else z
    y = _dropped(s, y)
    if c["residual"]:
        y = y + s["residual"].float()
    d = {}
    if c["out"]:
        d["out"] = y.to(dt)
    if c["packed"]:
        d["values"] = _rounded(y)
    if c["pre"]:
        d["pre"] = _rounded(z)
    return d


def _eight_bytes(M, C):
    """Rows in eight bits."""
    return M * -(-C // BLOCK) * (BLOCK + 1)


def work(case):
    """Eight-bit results are written once, and read once for the values in bfloat16 that a pass gives."""
    c, es = case, 4 if case["dtype"] == "fp32" else 2
    if c["op"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        if c["backward"]:
            n = M * N + M * K + 2 * K * N + (N if c["bias"] else 0)
            eight = _eight_bytes(M, K) + (_eight_bytes(M, N) if c["act"] != "none" else 0)
            return {"bytes": n * es + eight, "flops": 4.0 * M * K * N}
        n = (N if c["bias"] else 0) + M * N * (c["out"] + c["residual"])
        eight = _eight_bytes(M, K) + _eight_bytes(N, K) + (c["packed"] + c["pre"]) * (2 * _eight_bytes(M, N) + 2 * M * N)
        return {"bytes": n * es + eight, "flops": 2.0 * M * K * N}
    M, C = c["M"], c["C"]
    n = M * C
    if c["op"] == "pack":
        return {"bytes": n * es + 2 * _eight_bytes(M, C) + 2 * n, "flops": 4.0 * n}
    if c["backward"]:
        return {"bytes": n * es * (3 + c["residual"]) + C * es + 4 * C, "flops": 10.0 * n}
    eight = 2 * _eight_bytes(M, C) + 2 * n if c["packed"] else 0
    return {"bytes": n * es * (1 + 2 * c["residual"] + c["out"]) + C * es + eight, "flops": 4.0 * n}


# ---------------------------------------------------------------- the definitions, in float64


def _mul_hi_lo(a, m):
    """High and low 32 bits of a times m from 16-bit halves."""
    al, ah, ml, mh = a % 65536, a // 65536, m % 65536, m // 65536
    low, mid = al * ml, al * mh + ah * ml
    low = low + (mid % 65536) * 65536
    return ah * mh + mid // 65536 + low // 2 ** 32, low % 2 ** 32


def _exact_factor(s, n):
    """drop()'s factor of each of n elements, eight to a generator call."""
    place = (int(s["counter"].item()) + s["offset"]) % 2 ** 64
    T = _threshold(s["case"]["p"])
    i = torch.arange(-(-n // 8), dtype=torch.int64, device=s["counter"].device)
    ctr = [i % 2 ** 32, i // 2 ** 32, torch.full_like(i, place % 2 ** 32), torch.full_like(i, place // 2 ** 32)]
    for r in range(7):
        key = [(s["seed"] % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (s["seed"] // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32]
        (h0, l0), (h1, l1) = _mul_hi_lo(ctr[0], 0xD2511F53), _mul_hi_lo(ctr[2], 0xCD9E8D57)
        ctr = [torch.bitwise_xor(torch.bitwise_xor(h1, ctr[1]), key[0]), l1, torch.bitwise_xor(torch.bitwise_xor(h0, ctr[3]), key[1]), l0]
    f = torch.empty(i.numel(), 8, dtype=torch.float64, device=i.device)
    for j in range(8):
        f[:, j] = ((ctr[j // 2] // 65536 ** (j % 2)) % 65536 >= T).double()
    return f.reshape(-1)[:n] * (65536.0 / (65536 - T))


def _exact_round(v):
    """What rows of float64 become in eight bits: the steps of E4M3 written out."""
    M, C = v.shape
    b = torch.zeros(M, -(-C // BLOCK) * BLOCK, dtype=torch.float64, device=v.device)
    b[:, :C] = v
    b = b.reshape(M, -1, BLOCK)
    top = b.abs().max(2, keepdim=True).values
    # the smallest s with top <= 448 2^s
    s = torch.ceil(torch.log2(top / 448.0))
    s = torch.where(448.0 * torch.exp2(s) < top, s + 1, s)
    s = torch.where(448.0 * torch.exp2(s - 1) >= top, s - 1, s)
    scale = torch.exp2(s.clamp(-117, 119))
    u = b / scale
    # eight steps to each power of two, from 2^-6 down those of 2^-6
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6)))) / 8
    return (torch.round(u / step) * step * scale).reshape(M, -1)[:, :C]


def _exact_kept(t, C):
    q = t[0].double().reshape(t[0].shape[0], -1, BLOCK)
    return (q * torch.exp2(t[1].view(torch.uint8).double() - 127).unsqueeze(2)).reshape(t[0].shape[0], -1)[:, :C]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "pack":
        return {"values": _exact_round(s["x"].double())}
    if c["op"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        x = _exact_kept(s["x"], K)
        f = _exact_factor(s, M * N).reshape(M, N) if c["p"] else 1.0
        if c["backward"]:
            dz = s["g"].double() * f
            if c["p"]:  # a dropped gradient is 0 whatever it was
                dz = torch.where(f > 0, dz, torch.zeros_like(dz))
            if c["act"] == "relu":
                dz = dz * (_exact_kept(s["pre"], N) > 0)
            if c["act"] == "gelu":
                z = _exact_kept(s["pre"], N)
                dz = dz * (torch.special.ndtr(z) + z * torch.exp(z.square() / -2) / math.sqrt(2 * math.pi))
            d = {"dx": torch.matmul(dz, s["w"].double().t().contiguous()), "dw": torch.matmul(x.t().contiguous(), dz)}
            if c["bias"]:
                d["db"] = torch.ones(1, M, dtype=torch.float64, device=x.device).matmul(dz).reshape(N)
            return d
        z = torch.matmul(x, _exact_kept(s["w"], K).t().contiguous())
        if c["bias"]:
            z += s["b"].double()
        y = {"none": lambda t: t, "relu": lambda t: t.clamp(min=0), "gelu": lambda t: t * torch.special.ndtr(t)}[c["act"]](z) * f
        if c["residual"]:
            y = y + s["residual"].double()
        d = {"out": y} if c["out"] else {}
        if c["packed"]:
            d["values"] = _exact_round(y)
        if c["pre"]:
            d["pre"] = _exact_round(z)
        return d
    x = s["x"].double()
    if c["backward"]:
        d = (x.square().sum(1, keepdim=True) / c["C"] + EPS).sqrt()
        h, g = x / d, s["g"].double()
        a = g * s["gamma"].double()
        dx = (a - h * (torch.sum(a * h, 1, keepdim=True) / c["C"])) / d
        if c["residual"]:
            dx += s["residual"].double()
        return {"dx": dx, "dgamma": torch.sum(g * h, 0)}
    r = {}
    if c["residual"]:
        # the norm is of the sum as it is stored
        r["sum"] = x + s["residual"].double()
        x = r["sum"].to(s["x"].dtype).double()
    y = x / (x.square().sum(1, keepdim=True) / c["C"] + EPS).sqrt() * s["gamma"].double()
    if c["out"]:
        r["out"] = y
    if c["packed"]:
        r["values"] = _exact_round(y)
    return r
