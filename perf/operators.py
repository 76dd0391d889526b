"""Performance cases of the operators that train an AFNO block around its filter, one call through a
public entry point per case, with the operators' plain forms.

Operators ("op" of a case, "backward" its direction):
  linear      out = drop(act(x w + b)) + residual; the gradients dx, dw, db of drop(act(x w + b)).
  layer_norm  out = LN(x + residual) and the sum; the gradients dx, dgamma, dbeta.
  dropout     out = drop(x) + residual; the gradient dx.
drop() keeps element e (its flat index) where a 16-bit number of the counter-based generator Philox4x32
with seven rounds is at least T = 65536 p rounded, and scales by 65536 / (65536 - T).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


def _linear(name, M, K, N, dtype, backward=False, act="gelu", p=0.0, residual=False, bias=True, pre=False):
    return {"name": name, "op": "linear", "backward": backward, "M": M, "K": K, "N": N, "dtype": dtype, "act": act,
            "p": p, "residual": residual, "bias": bias, "pre": pre}


def _norm(name, M, C, dtype, backward=False, residual=False):
    return {"name": name, "op": "layer_norm", "backward": backward, "M": M, "C": C, "dtype": dtype, "residual": residual}


def _drop(name, n, dtype, backward=False, p=0.1, residual=False):
    return {"name": name, "op": "dropout", "backward": backward, "n": n, "dtype": dtype, "p": p, "residual": residual}


def listed():
    return [
        # one token through the MLP's first product: a probe of one grid point, where latency and the weights count
        _linear("linear_1_token_bf16", 1, 1024, 4096, "bf16"),
        # a training step of a toy model on a 16 x 32 grid: launches count
        _linear("linear_16x32_fp32", 512, 64, 256, "fp32", p=0.1, pre=True),
        # the MLP's first product in training on the 180 x 360 grid, 4,096 hidden units for 1,024 channels
        _linear("linear_up_180x360_bf16", 64800, 1024, 4096, "bf16", p=0.1, pre=True),
        # its second product, back to the channels and onto the residual stream
        _linear("linear_down_180x360_bf16", 64800, 4096, 1024, "bf16", act="none", p=0.1, residual=True),
        # a projection of sizes that no tile divides, on a regional 45 x 91 grid
        _linear("linear_ragged_bf16", 4095, 333, 77, "bf16", act="relu"),
        # the gradient of the first product
        _linear("linear_backward_180x360_bf16", 64800, 1024, 4096, "bf16", backward=True, p=0.1),
        # training at full precision on a 2.5-degree grid
        _linear("linear_backward_72x144_fp32", 10368, 384, 1536, "fp32", backward=True),
        # the sum of the residual stream and the filter's output, and its norm
        _norm("layer_norm_180x360_bf16", 64800, 1024, "bf16", residual=True),
        # the gradient through that norm, onto the gradient of the residual stream
        _norm("layer_norm_backward_180x360_bf16", 64800, 1024, "bf16", backward=True, residual=True),
        # an odd number of channels at full precision
        _norm("layer_norm_backward_odd_fp32", 5187, 333, "fp32", backward=True),
        # dropout of a branch on its way into the residual stream
        _drop("dropout_180x360_bf16", 64800 * 1024, "bf16", residual=True),
        # the gradient of a small field of odd size
        _drop("dropout_backward_odd_fp32", 45 * 91 * 77, "fp32", backward=True, p=0.25),
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
        op = rng.choices(["linear", "layer_norm", "dropout"], [6, 3, 1])[0]
        dtype = "bf16" if rng.random() < 0.65 else "fp32"
        backward, residual = rng.random() < 0.4, rng.random() < 0.5
        M = _log(rng, 1, 64800)
        p = 0.0 if rng.random() < 0.4 else round(rng.uniform(0.02, 0.6), 3)
        if op == "linear":
            K, N = _width(rng, 8, 4096), _width(rng, 8, 4096)
            act = rng.choice(["none", "relu", "gelu", "gelu"])
            c = _linear("", M, K, N, dtype, backward, act, p, residual and not backward, rng.random() < 0.85,
                        act != "none" and not backward and rng.random() < 0.5)
            # no dearer than the largest case listed, which is in bf16 and has 1.1e12 operations
            if (4.0 if backward else 2.0) * M * K * N > (1.0e12 if dtype == "bf16" else 3.0e11):
                continue
        elif op == "layer_norm":
            c = _norm("", M, _width(rng, 8, 4096), dtype, backward, residual)
            if M * c["C"] > 64800 * 1024:
                continue
        else:
            c = _drop("", _log(rng, 1000, 64800 * 1024), dtype, backward, p or 0.1, residual and not backward)
        del c["name"]
        return c


def prepare(case, seed):
    c, dt, dev = case, DTYPES[case["dtype"]], torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(1000003 * int(seed) + 29)

    def normal(*shape, std=1.0, mean=0.0):
        return (mean + std * torch.randn(*shape, generator=g, device=dev)).to(dt)

    s = {"case": dict(c)}
    if c.get("p"):
        # the run's seed, this operator's place in the model, and the training step on the device
        s["seed"], s["offset"] = 0x9E3779B97F4A7C15 * (int(seed) + 1) % 2 ** 64, 3 << 40
        s["counter"] = torch.tensor([1000 + int(seed) % 1000], dtype=torch.int64, device=dev)
    if c["op"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        # activations whose channels differ in scale, weights that keep it
        s["x"] = (torch.randn(M, K, generator=g, device=dev) * (0.5 + torch.rand(K, generator=g, device=dev))).to(dt)
        s["w"] = normal(K, N, std=1.0 / math.sqrt(K))
        s["b"] = normal(N, std=0.1) if c["bias"] else None
        if c["backward"]:
            s["g"] = normal(M, N)
            s["pre"] = None
            if c["act"] != "none":
                z = s["x"] @ s["w"]
                s["pre"] = z + s["b"] if c["bias"] else z
        if c["residual"]:
            s["residual"] = normal(M, N)
    elif c["op"] == "layer_norm":
        M, C = c["M"], c["C"]
        s["gamma"], s["beta"] = normal(C, std=0.1, mean=1.0), normal(C, std=0.1)
        s["x"] = (0.2 + torch.randn(M, C, generator=g, device=dev) * (0.5 + 1.5 * torch.rand(C, generator=g, device=dev))).to(dt)
        if c["residual"]:
            s["residual"] = normal(M, C)
        if c["backward"]:
            s["g"] = normal(M, C)
    else:
        s["x"] = normal(c["n"])
        if c["residual"]:
            s["residual"] = normal(c["n"])
    return s


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2208_05419_amd as afno
    c = s["case"]
    rng = {"p": c["p"], "seed": s["seed"], "offset": s["offset"], "counter": s["counter"]} if c.get("p") else {}
    if c["op"] == "linear":
        if c["backward"]:
            d = afno.linear_backward(s["g"], s["x"], s["w"], pre=s["pre"], activation=c["act"], bias=c["bias"], **rng)
            return {k: v for k, v in d.items() if v is not None}
        out = torch.empty(c["M"], c["N"], dtype=s["x"].dtype, device=s["x"].device)
        pre = torch.empty_like(out) if c["pre"] else None
        afno.linear_forward(s["x"], s["w"], s["b"], activation=c["act"], residual=s.get("residual"), out=out, pre=pre, **rng)
        return {"out": out, "pre": pre} if c["pre"] else {"out": out}
    if c["op"] == "layer_norm":
        if c["backward"]:
            return afno.layer_norm_backward(s["g"], s["x"], s["gamma"], eps=EPS, gsum=s.get("residual"))
        v = torch.empty_like(s["x"]) if c["residual"] else None
        out = afno.layer_norm_forward(s["x"], s["gamma"], s["beta"], eps=EPS, residual=s.get("residual"), sum_out=v)
        return {"out": out, "sum": v} if c["residual"] else {"out": out}
    if c["backward"]:
        return {"dx": afno.dropout_backward(s["x"], **rng)}
    return {"out": afno.dropout_forward(s["x"], residual=s.get("residual"), **rng)}


# ---------------------------------------------------------------- plain forms, in float32


def _threshold(p):
    return int(np.rint(float(np.float32(p)) * 65536.0))


def _keep(s, n):
    """Which of n elements the generator keeps."""
    low = 0xFFFFFFFF
    group = torch.arange((n + 7) // 8, dtype=torch.int64, device=s["x"].device)
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


def _run_plain(s):
    c, dt = s["case"], s["x"].dtype
    x = s["x"].float()
    if c["op"] == "linear":
        w = s["w"].float()
        if c["backward"]:
            dz = _dropped(s, s["g"].float())
            if c["act"] == "relu":
                dz = torch.where(s["pre"].float() > 0, dz, 0.0)
            elif c["act"] == "gelu":
                z = s["pre"].float()
                dz = dz * (0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi)))
            d = {"dx": (dz @ w.t()).to(dt), "dw": (x.t() @ dz).to(dt)}
            return {**d, "db": dz.sum(0).to(dt)} if c["bias"] else d
        z = x @ w
        if c["bias"]:
            z = z + s["b"].float()
        y = torch.relu(z) if c["act"] == "relu" else 0.5 * z * torch.erfc(z * -math.sqrt(0.5)) if c["act"] == "gelu" else z
        y = _dropped(s, y)
        if c["residual"]:
            y = y + s["residual"].float()
        return {"out": y.to(dt), "pre": z.to(dt)} if c["pre"] else {"out": y.to(dt)}
    if c["op"] == "dropout":
        y = _dropped(s, x)
        if c["residual"]:
            y = y + s["residual"].float()
        return {"dx": y.to(dt)} if c["backward"] else {"out": y.to(dt)}
    if not c["backward"] and c["residual"]:
        v = (x + s["residual"].float()).to(dt)
        x = v.float()
    centred = x - x.mean(-1, keepdim=True)
    rstd = torch.rsqrt((centred * centred).mean(-1, keepdim=True) + EPS)
    xh = centred * rstd
    if not c["backward"]:
        out = (xh * s["gamma"].float() + s["beta"].float()).to(dt)
        return {"out": out, "sum": v} if c["residual"] else {"out": out}
    g = s["g"].float()
    a = g * s["gamma"].float()
    dx = rstd * (a - a.mean(-1, keepdim=True) - xh * (a * xh).mean(-1, keepdim=True))
    if c["residual"]:
        dx = dx + s["residual"].float()
    return {"dx": dx.to(dt), "dgamma": (g * xh).sum(0), "dbeta": g.sum(0)}


def work(case):
    c, es = case, 4 if case["dtype"] == "fp32" else 2
    if c["op"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        if c["backward"]:
            n = M * N * (2 if c["act"] != "none" else 1) + 2 * (M * K + K * N) + (N if c["bias"] else 0)
            return {"bytes": n * es, "flops": 4.0 * M * K * N}
        n = M * K + K * N + (N if c["bias"] else 0) + M * N * (1 + c["pre"] + c["residual"])
        return {"bytes": n * es, "flops": 2.0 * M * K * N}
    if c["op"] == "layer_norm":
        n, C = c["M"] * c["C"], c["C"]
        if c["backward"]:
            return {"bytes": n * es * (3 + c["residual"]) + C * es + 8 * C, "flops": 14.0 * n}
        return {"bytes": n * es * (2 + 2 * c["residual"]) + 2 * C * es, "flops": 8.0 * n}
    return {"bytes": c["n"] * es * (2 + c["residual"]), "flops": 2.0 * c["n"]}


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
    i = torch.arange(-(-n // 8), dtype=torch.int64, device=s["x"].device)
    ctr = [i % 2 ** 32, i // 2 ** 32, torch.full_like(i, place % 2 ** 32), torch.full_like(i, place // 2 ** 32)]
    for r in range(7):
        key = [(s["seed"] % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (s["seed"] // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32]
        (h0, l0), (h1, l1) = _mul_hi_lo(ctr[0], 0xD2511F53), _mul_hi_lo(ctr[2], 0xCD9E8D57)
        ctr = [torch.bitwise_xor(torch.bitwise_xor(h1, ctr[1]), key[0]), l1, torch.bitwise_xor(torch.bitwise_xor(h0, ctr[3]), key[1]), l0]
    f = torch.empty(i.numel(), 8, dtype=torch.float64, device=i.device)
    for j in range(8):
        f[:, j] = ((ctr[j // 2] // 65536 ** (j % 2)) % 65536 >= T).double()
    return f.reshape(-1)[:n] * (65536.0 / (65536 - T))


def exact(case, seed):
    c, s = case, prepare(case, seed)
    x = s["x"].double()
    if c["op"] == "linear":
        M, N = c["M"], c["N"]
        f = _exact_factor(s, M * N).reshape(M, N) if c["p"] else 1.0
        if c["backward"]:
            dz = s["g"].double() * f
            if c["p"]:  # a dropped gradient is 0 whatever it was
                dz = torch.where(f > 0, dz, torch.zeros_like(dz))
            if c["act"] == "relu":
                dz = dz * (s["pre"] > 0)
            if c["act"] == "gelu":
                z = s["pre"].double()
                dz = dz * (torch.special.ndtr(z) + z * torch.exp(z.square() / -2) / math.sqrt(2 * math.pi))
            d = {"dx": torch.matmul(dz, s["w"].double().t().contiguous()), "dw": torch.matmul(x.t().contiguous(), dz)}
            if c["bias"]:
                d["db"] = torch.ones(1, M, dtype=torch.float64, device=x.device).matmul(dz).reshape(N)
            return d
        z = torch.matmul(x, s["w"].double())
        if c["bias"]:
            z += s["b"].double()
        y = {"none": lambda t: t, "relu": lambda t: t.clamp(min=0), "gelu": lambda t: t * torch.special.ndtr(t)}[c["act"]](z) * f
        if c["residual"]:
            y = y + s["residual"].double()
        return {"out": y, "pre": z} if c["pre"] else {"out": y}
    if c["op"] == "dropout":
        y = x * _exact_factor(s, c["n"])
        if c["residual"]:
            y += s["residual"].double()
        return {"dx": y} if c["backward"] else {"out": y}
    if c["backward"]:
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        sd = (var + EPS).sqrt()
        xh, g = (x - mean) / sd, s["g"].double()
        a = g * s["gamma"].double()
        dx = (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True)) / sd
        if c["residual"]:
            dx += s["residual"].double()
        return {"dx": dx, "dgamma": torch.sum(g * xh, 0), "dbeta": torch.sum(g, 0)}
    v = None
    if c["residual"]:
        # the norm is of the sum as it is stored
        v = x + s["residual"].double()
        x = v.to(s["x"].dtype).double()
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    out = (x - mean) / (var + EPS).sqrt() * s["gamma"].double() + s["beta"].double()
    return {"out": out, "sum": v} if c["residual"] else {"out": out}
