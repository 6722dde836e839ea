"""Measured cases of the operators of a training step of adapters beside frozen projections.

* Layer norm with a block's modulation or a plain weight (`sol_layernorm`, `sol_layernorm_backward`): BF16 forward with
  the row statistics, and the gradients of x and, summed over each sample's rows, of scale and shift.
* Low-rank adapters of many requests at once (`sol_lora_apply`, `sol_lora_backward`): y += s (x A^T) B^T where every run
  of rows has an adapter of its own or none, and the gradients of x, A and B.
* AdamW over many tensors at once (`sol_adamw_plan`, `sol_adamw_step`) with 32-bit states or 8-bit ones: blocks of 32
  values under a power of two, the first moment in E4M3, the second in E5M2, rounded up or down at random in proportion.

Every operator has its plain form here (elementary torch operations in 32 bits) and, with `own` true, the call a user makes.
"""
import math

import numpy as np
import torch

own = False


DEV = "cuda"
EPS = 1e-6                                   # of the norms
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-4, 0.9, 0.999, 1e-8, 0.01
SEED, STEPS = 20260917, 100                  # seed of the rounding, steps that the states have behind them
GROUP = 32                                   # values under one scale


def _binding():
    from paper_2604_06916_b200 import binding as b
    return b


# ------------------------------------------------------------------------------------------------ cases
# A, B of the four linears of one FLUX double-stream block's stream at rank 32: 3072 -> 9216, 3072, 12288 and 12288 -> 3072
FLUX_ADAPTERS = "98304 294912 98304 98304 98304 393216 393216 98304"


def listed():
    return [
        # the text tokens of one SD3.5 sample
        {"name": "norm 333x2432", "op": "norm", "back": False, "M": 333, "K": 2432, "rows": 333, "one": True, "shift": True},
        # a FLUX block's modulated norm, eight samples at 1024 pixels
        {"name": "norm 36864x3072 8 samples", "op": "norm", "back": False, "M": 36864, "K": 3072, "rows": 4608, "one": True, "shift": True},
        # its gradients for two samples
        {"name": "norm grad 9216x3072 2 samples", "op": "norm", "back": True, "M": 9216, "K": 3072, "rows": 4608, "one": True, "shift": True},
        # a norm with a weight and a bias over all tokens of three SD3.5 samples
        {"name": "norm grad 13287x2432 weight", "op": "norm", "back": True, "M": 13287, "K": 2432, "rows": 13287, "one": False, "shift": True},
        # one modulation linear for eight requests, each with an adapter of its own
        {"name": "lora 8 requests of 1 row", "op": "lora", "back": False, "lens": "1 1 1 1 1 1 1 1", "ids": "3 0 5 1 7 2 6 4", "n": 8, "pad": 0,
         "r": 32, "K": 3072, "N": 18432, "dx": False},
        # candidates of three policies and of the base model in one batch, 512-pixel samples, ragged text, through a FLUX qkv projection
        {"name": "lora 17003 rows 3 adapters", "op": "lora", "back": False, "lens": "1536 3072 1411 1536 4375 1 4608 464", "ids": "0 1 2 -1 0 1 2 0", "n": 3,
         "pad": 21, "r": 32, "K": 3072, "N": 9216, "dx": False},
        # stage 2: one adapter, two samples at 1024 pixels, gradients through the same projection
        {"name": "lora grad 9216 rows", "op": "lora", "back": True, "lens": "9216", "ids": "0", "n": 1, "pad": 0, "r": 32, "K": 3072, "N": 9216, "dx": True},
        # two adapters, ragged samples and one without an adapter, an SD3.5 output projection at rank 16
        {"name": "lora grad 5 ragged r16", "op": "lora", "back": True, "lens": "333 1024 77 1 2049", "ids": "1 0 1 1 -1", "n": 2, "pad": 13, "r": 16,
         "K": 2432, "N": 2432, "dx": True},
        # the adapter of one FLUX output projection, with the BF16 copy that the linears read
        {"name": "adamw32 one adapter", "op": "adamw", "bits": 32, "sizes": "98304 98304", "count": 2, "p16": False, "g16": False, "copy": True},
        # the adapters of 19 FLUX double-stream blocks, both streams
        {"name": "adamw32 304 tensors", "op": "adamw", "bits": 32, "sizes": FLUX_ADAPTERS, "count": 304, "p16": False, "g16": False, "copy": True},
        # the same with states in 8 bits
        {"name": "adamw8 304 tensors", "op": "adamw", "bits": 8, "sizes": FLUX_ADAPTERS, "count": 304, "p16": False, "g16": False, "copy": True},
        # the full weights of an SD3.5 block in BF16, odd biases beside them, states in 8 bits
        {"name": "adamw8 block in bf16", "op": "adamw", "bits": 8, "sizes": "17743872 7296 5914624 2432 23658496 9728 23658496 2432 35467", "count": 9,
         "p16": True, "g16": True, "copy": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm grad", "lora", "lora grad", "adamw"])
    if op.startswith("norm"):
        K = 8 * _log(rng, 8, 1500)
        M = _log(rng, 1, 40000)
        while M * K > (36864 if op == "norm" else 9216) * 3072:
            M = max(1, M // 2)
        return {"op": "norm", "back": op == "norm grad", "M": M, "K": K, "rows": -(-M // _log(rng, 1, 16)), "one": rng.random() < 0.6,
                "shift": rng.random() < 0.8}
    if op.startswith("lora"):
        K, N, r = 8 * _log(rng, 16, 1600), 8 * _log(rng, 16, 2400), 8 * rng.randint(1, 8)
        n = _log(rng, 1, 8)
        lens = [_log(rng, 1, 5000) for _ in range(_log(rng, 1, 12))]
        # the plain form pads every request to the longest
        while len(lens) * max(lens) * (K + N) > 17003 * 12288 * (2 if op == "lora" else 1):
            lens = [max(1, v // 2) for v in lens]
        ids = [rng.randint(-1, n - 1) for _ in lens]
        ids[rng.randrange(len(ids))] = n - 1
        return {"op": "lora", "back": op == "lora grad", "lens": " ".join(map(str, lens)), "ids": " ".join(map(str, ids)), "n": n,
                "pad": rng.choice([0, 0, rng.randint(1, 200)]), "r": r, "K": K, "N": N, "dx": op == "lora grad" and rng.random() < 0.7}
    sizes = [_log(rng, 1, 4000000) for _ in range(_log(rng, 1, 300))]
    while sum(sizes) > 40000000:
        sizes = [max(1, v // 2) for v in sizes]
    p16 = rng.random() < 0.4
    return {"op": "adamw", "bits": rng.choice([8, 32]), "sizes": " ".join(map(str, sizes)), "count": len(sizes), "p16": p16, "g16": p16 or rng.random() < 0.3,
            "copy": not p16 and rng.random() < 0.5}


def _ints(text):
    return [int(v) for v in text.split()]


def _sizes(case):
    some = _ints(case["sizes"])
    return [some[i % len(some)] for i in range(case["count"])]


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed) * 6361 + 29)
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    st = {"case": case}
    if case["op"] == "norm":
        M, K, S = case["M"], case["K"], -(-case["M"] // case["rows"])
        # a residual stream: every channel has its own size and offset
        st["x"] = (randn(M, K) * torch.exp(0.5 * randn(K)) + 0.3 * randn(K)).to(torch.bfloat16)
        st["scale"] = ((0.0 if case["one"] else 1.0) + 0.2 * randn(S, K)).to(torch.bfloat16)
        st["shift"] = (0.2 * randn(S, K)).to(torch.bfloat16) if case["shift"] else None
        if case["back"]:
            st["dy"] = randn(M, K).to(torch.bfloat16)
            x = st["x"].double()
            mu = x.mean(1)
            st["stats"] = torch.stack((mu, (x.var(1, correction=0) + EPS).rsqrt()), dim=1).float()
        return st
    if case["op"] == "lora":
        K, N, r, n, lens = case["K"], case["N"], case["r"], case["n"], _ints(case["lens"])
        M = sum(lens) + case["pad"]
        st["x"] = randn(M, K).to(torch.bfloat16)
        st["a"] = (randn(n, r, K) * r ** -0.5).to(torch.bfloat16)
        st["b"] = (randn(n, N, r) * 0.02).to(torch.bfloat16)
        st["scaling"] = torch.full((n,), 2.0, device=DEV) * (1.0 + 0.5 * torch.arange(n, device=DEV))
        st["offsets"] = torch.tensor([0] + np.cumsum(lens).tolist(), dtype=torch.int32, device=DEV)
        st["ids"] = torch.tensor(_ints(case["ids"]), dtype=torch.int32, device=DEV)
        st["longest"] = max(lens)
        if not case["back"]:
            st["y"] = randn(M, N).to(torch.bfloat16)       # the shared projection's output
            return st
        st["dy"] = randn(M, N).to(torch.bfloat16)
        st["dx"] = randn(M, K).to(torch.bfloat16) if case["dx"] else None   # the shared projection's gradient
        # what the forward call leaves: t = x A^T in two BF16 parts side by side
        t = torch.zeros((M, r), device=DEV)
        for i, a in enumerate(_ints(case["ids"])):
            rows = slice(sum(lens[:i]), sum(lens[:i + 1]))
            if a >= 0:
                t[rows] = st["x"][rows].float() @ st["a"][a].float().T
        hi = t.to(torch.bfloat16)
        st["t"] = torch.cat((hi, (t - hi.float()).to(torch.bfloat16)), dim=1).contiguous()
        return st
    sizes = _sizes(case)
    # every tensor starts on a multiple of 128 values of the flat buffers; what lies between stays as it is
    starts = np.concatenate(([0], np.cumsum([-(-v // 128) * 128 for v in sizes])))
    total = int(starts[-1])
    st["sizes"], st["starts"], st["total"], st["steps"] = sizes, [int(v) for v in starts[:-1]], total, STEPS
    st["p"] = (0.02 * randn(total)).to(torch.bfloat16 if case["p16"] else torch.float32)
    # gradients of different tensors differ in size, those of a tensor spread over a few powers of ten
    size = torch.exp(1.5 * randn(len(sizes))).repeat_interleave(torch.tensor([-(-v // 128) * 128 for v in sizes], device=DEV), output_size=total)
    spread = 1e-4 * size * torch.exp(randn(total))
    st["g"] = (spread * randn(total)).to(torch.bfloat16 if case["g16"] else torch.float32)
    m, v = 0.3 * spread * randn(total), (spread * (0.5 + torch.rand(total, generator=g, device=DEV))).square()
    st["copy"] = st["p"].to(torch.bfloat16) if case["copy"] else None
    if case["bits"] == 8:
        st["m"], st["ms"] = _encode(m, 3, None)
        st["v"], st["vs"] = _encode(v, 2, None)
    else:
        st["m"], st["v"] = m, v
    if case["bits"] == 8 or case["p16"]:
        at, which = torch.arange(total, device=DEV), torch.zeros(total, dtype=torch.int64, device=DEV)
        which[torch.tensor(st["starts"], device=DEV)] = 1
        which = which.cumsum(0) - 1
        st["which"], st["within"] = which, at - torch.tensor(st["starts"], device=DEV)[which]
    if own:    # the plan: the same tensors as above, laid out once for the calls of a training loop
        cut = lambda flat, unit=1: [flat[s // unit:s // unit + -(-v // unit)] for s, v in zip(st["starts"], sizes)]  # noqa: E731
        st["plan"] = _binding().sol_adamw_plan(
            cut(st["p"]), cut(st["g"]), copies=cut(st["copy"]) if case["copy"] else None, state_bits=case["bits"], step=STEPS,
            states={"m": cut(st["m"]), "v": cut(st["v"])} if case["bits"] == 32 else
            {"m": cut(st["m"]), "v": cut(st["v"]), "m_scale": cut(st["ms"], GROUP), "v_scale": cut(st["vs"], GROUP)})
    return st


# ------------------------------------------------------------------------------------------------ the calls
def run(st):
    c = st["case"]
    if c["op"] == "norm":
        if own:
            return _own_norm(st)
        return _plain_norm_grad(st) if c["back"] else _plain_norm(st)
    if c["op"] == "lora":
        if own:
            return _own_lora(st)
        return _plain_lora_grad(st) if c["back"] else _plain_lora(st)
    return _own_adamw(st) if own else _plain_adamw(st)


def _own_norm(st):
    b, c = _binding(), st["case"]
    offset = 1.0 if c["one"] else 0.0
    if not c["back"]:
        return b.sol_layernorm(st["x"], st["scale"], st["shift"], c["rows"], eps=EPS, scale_offset=offset, with_stats=True)
    dx, dscale, dshift = b.sol_layernorm_backward(st["dy"], st["x"], st["stats"], st["scale"], c["rows"], scale_offset=offset,
                                                  with_shift=c["shift"])
    return (dx, dscale, dshift) if c["shift"] else (dx, dscale)


def _own_lora(st):
    b, c = _binding(), st["case"]
    if not c["back"]:
        return b.sol_lora_apply(st["x"], st["a"], st["b"], st["scaling"], st["offsets"], st["ids"], st["y"])
    da, db = b.sol_lora_backward(st["dy"], st["x"], st["t"], st["a"], st["b"], st["scaling"], st["offsets"], st["ids"], dx=st["dx"])
    return (da, db, st["dx"]) if c["dx"] else (da, db)


def _own_adamw(st):
    c = st["case"]
    _binding().sol_adamw_step(st["plan"], lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY,
                              seed=SEED if c["bits"] == 8 or c["p16"] else None)
    return _adamw_outputs(st)


def _adamw_outputs(st):
    """The updated tensors; what is held in 8 bits as the values it stands for: E4M3 or E5M2 under a power of two per 32."""
    out = {"p": st["p"], "m": st["m"], "v": st["v"]}
    if st["case"]["bits"] == 8:
        out["m"], out["v"] = st["m"].view(torch.float8_e4m3fn), st["v"].view(torch.float8_e5m2)
        out["ms"], out["vs"] = st["ms"].view(torch.float8_e8m0fnu), st["vs"].view(torch.float8_e8m0fnu)
    if st["case"]["copy"]:
        out["copy"] = st["copy"]
    return out


# ------------------------------------------------------------------------------------------------ plain forms
def _by_sample(t, rows):
    """[M, K] -> [S, rows, K], the last sample filled up with zeros."""
    S = -(-t.shape[0] // rows)
    if S * rows != t.shape[0]:
        t = torch.cat((t, t.new_zeros((S * rows - t.shape[0], t.shape[1]))))
    return t.reshape(S, rows, t.shape[1])


def _plain_norm(st):
    c = st["case"]
    x = st["x"].float()
    mu = x.mean(1, keepdim=True)
    d = x - mu
    rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    gain = st["scale"].float() + (1.0 if c["one"] else 0.0)
    y = _by_sample(d * rstd, c["rows"]) * gain[:, None, :]
    if st["shift"] is not None:
        y = y + st["shift"].float()[:, None, :]
    return y.reshape(-1, c["K"])[:c["M"]].to(torch.bfloat16), torch.cat((mu, rstd), dim=1)


def _plain_norm_grad(st):
    c = st["case"]
    M, K, rows = c["M"], c["K"], c["rows"]
    mu, rstd = st["stats"][:, :1], st["stats"][:, 1:]
    xhat = (st["x"].float() - mu) * rstd
    dy = _by_sample(st["dy"].float(), rows)
    gain = st["scale"].float() + (1.0 if c["one"] else 0.0)
    w = (dy * gain[:, None, :]).reshape(-1, K)[:M]
    dx = rstd * (w - w.mean(1, keepdim=True) - xhat * (w * xhat).mean(1, keepdim=True))
    out = (dx.to(torch.bfloat16), (dy * _by_sample(xhat, rows)).sum(1))
    return out + (dy.sum(1),) if c["shift"] else out


def _requests(st):
    """Rows of each request [S, longest], which of them exist and belong to an adapter, and the adapters (0 for none)."""
    first, behind = st["offsets"][:-1].long(), st["offsets"][1:].long()
    at = first[:, None] + torch.arange(st["longest"], device=DEV)
    there = (at < behind[:, None]) & (st["ids"] >= 0)[:, None]
    return torch.where(there, at, 0), there, st["ids"].long().clamp(min=0)


def _plain_lora(st):
    at, there, ids = _requests(st)
    t = torch.bmm(st["x"].float()[at], st["a"].float()[ids].transpose(1, 2))
    add = torch.bmm(t, st["b"].float()[ids].transpose(1, 2)) * st["scaling"][ids][:, None, None]
    rows = at[there]
    st["y"][rows] = (st["y"][rows].float() + add[there]).to(torch.bfloat16)
    return st["y"]


def _plain_lora_grad(st):
    c = st["case"]
    n, r, K, N = c["n"], c["r"], c["K"], c["N"]
    at, there, ids = _requests(st)
    a, b, s = st["a"].float()[ids], st["b"].float()[ids], st["scaling"][ids][:, None, None]
    mask = there[:, :, None].float()
    dy, x = st["dy"].float()[at] * mask, st["x"].float()[at] * mask
    t = (st["t"][:, :r].float() + st["t"][:, r:].float())[at] * mask
    dt = torch.bmm(dy, b) * s
    pick = (ids == torch.arange(n, device=DEV)[:, None]).float()     # which request counts for which adapter
    da = (pick @ torch.bmm(dt.transpose(1, 2), x).reshape(-1, r * K)).reshape(n, r, K)
    db = (pick @ (torch.bmm(dy.transpose(1, 2), t) * s).reshape(-1, N * r)).reshape(n, N, r)
    if not c["dx"]:
        return da, db
    rows = at[there]
    st["dx"][rows] = (st["dx"][rows].float() + torch.bmm(dt, a)[there]).to(torch.bfloat16)
    return da, db, st["dx"]


WORD = 0xFFFFFFFF


def _mix(x):
    """A 32-bit integer (in 64 bits) mixed by two products and three shifts."""
    x = (x ^ (x >> 16)) & WORD
    x = (x * 0x7FEB352D) & WORD
    x = x ^ (x >> 15)
    x = (x * 0x846CA68B) & WORD
    return x ^ (x >> 16)


def _noise(st, step):
    """32 random bits per value, from the seed, the step, the tensor's number and the place in it."""
    h = 0
    for word in (SEED & WORD, SEED >> 32, step & WORD, step >> 32):
        h = _mix(h ^ ((word + 0x9E3779B9) & WORD))
    h = _mix(h ^ ((st["which"] + 0x9E3779B9) & WORD))
    return _mix(h ^ st["within"])


def _round_bits(bits, drop, noise):
    """Integer `bits` without the last `drop`: rounded up with the chance that they stand for, or to nearest (ties to even)."""
    if noise is None:
        return (bits + ((1 << (drop - 1)) - 1) + ((bits >> drop) & 1)) >> drop
    return (bits + (noise << (drop - 16)) + (1 << (drop - 16) >> 1)) >> drop


def _encode(v, mantissa, noise):
    """8-bit floats of 1 sign bit and `mantissa` mantissa bits in blocks of 32 under a power of two that takes the largest to
    [2^7, 2^8) (three mantissa bits) or [2^14, 2^15) (two): codes and the powers' exponents + 127."""
    top, shift = (7, 2.0 ** -120) if mantissa == 3 else (14, 2.0 ** -112)
    size = v.abs()
    fine = size < math.inf
    most = torch.where(fine, size, 0.0).reshape(-1, GROUP).amax(1)
    e = ((most.view(torch.int32) >> 23) - top).clamp(min=1)
    small = size * ((254 - e) << 23).view(torch.float32).repeat_interleave(GROUP) * shift   # its bits are the code's, further down
    drop = 23 - mantissa
    code = _round_bits(small.view(torch.int32), drop, noise)
    code = torch.where(fine, code, 127) | ((v.view(torch.int32) >> 31) & 1) << 7
    return code.to(torch.uint8), e.to(torch.uint8)


def _decode(code, e, mantissa):
    code = code.int()
    size = ((code & 127) << (23 - mantissa)).view(torch.float32) * (2.0 ** 120 if mantissa == 3 else 2.0 ** 112)
    size = torch.where((code & 127) == 127, math.nan, size * (e.int() << 23).view(torch.float32).repeat_interleave(GROUP))
    return torch.where(code > 127, -size, size)


def _plain_adamw(st):
    c = st["case"]
    st["steps"] += 1
    eight = c["bits"] == 8
    noise = _noise(st, st["steps"]) if eight or c["p16"] else None
    if noise is not None:
        live = st["within"] < torch.tensor(st["sizes"], device=DEV)[st["which"]]
    else:
        ends = torch.tensor([a + b for a, b in zip(st["starts"], st["sizes"])], device=DEV)
        live = torch.arange(st["total"], device=DEV) < ends.repeat_interleave(
            torch.tensor([-(-v // 128) * 128 for v in st["sizes"]], device=DEV), output_size=st["total"])
    p, g = st["p"].float(), st["g"].float()
    m, v = (_decode(st["m"], st["ms"], 3), _decode(st["v"], st["vs"], 2)) if eight else (st["m"], st["v"])
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    size = LR / (1.0 - BETA1 ** st["steps"])
    p = p * (1.0 - LR * DECAY) - m * size / (torch.sqrt(v) * (1.0 / math.sqrt(1.0 - BETA2 ** st["steps"])) + ADAM_EPS)
    if c["p16"]:
        low = (noise * 0x9E3779B1 >> 16) & 0xFFFF
        short = (_round_bits(p.view(torch.int32).long() & WORD, 16, low) << 16).to(torch.int32).view(torch.float32)
        p = torch.where(p.isfinite(), short, p)
    st["p"].copy_(torch.where(live, p, st["p"].float()))
    if c["copy"]:
        st["copy"].copy_(torch.where(live, p.to(torch.bfloat16), st["copy"]))
    if not eight:
        st["m"].copy_(torch.where(live, m, st["m"]))
        st["v"].copy_(torch.where(live, v, st["v"]))
        return _adamw_outputs(st)
    # a block's scale is that of its own tensor's values; blocks behind a tensor's end keep what they hold
    noise = noise.int()
    for name, now, mantissa, bits in (("m", m, 3, noise & 0xFFFF), ("v", v, 2, (noise >> 16) & 0xFFFF)):
        code, e = _encode(torch.where(live, now, 0.0), mantissa, bits)
        st[name].copy_(torch.where(live, code, st[name]))
        st[name + "s"].copy_(torch.where(live[::GROUP], e, st[name + "s"]))
    return _adamw_outputs(st)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] == "norm":
        M, K, S = case["M"], case["K"], -(-case["M"] // case["rows"])
        if case["back"]:
            return {"bytes": 6 * M * K + 8 * M + 2 * S * K + (8 if case["shift"] else 4) * S * K, "flops": 14 * M * K}
        return {"bytes": 4 * M * K + 8 * M + (4 if case["shift"] else 2) * S * K, "flops": 8 * M * K}
    if case["op"] == "lora":
        K, N, r = case["K"], case["N"], case["r"]
        ids = _ints(case["ids"])
        rows = sum(v for v, a in zip(_ints(case["lens"]), ids) if a >= 0)
        weights = 2 * len({a for a in ids if a >= 0}) * r * (K + N)
        if case["back"]:
            products = 3 if not case["dx"] else 4
            flops = 2 * rows * r * (2 * N + (products - 2) * K)
            return {"bytes": rows * (2 * K + 2 * N + 4 * r + (4 * K if case["dx"] else 0)) + weights + 4 * case["n"] * r * (K + N), "flops": flops}
        return {"bytes": rows * (2 * K + 4 * N) + weights, "flops": 2 * rows * r * (K + N)}
    n = sum(_sizes(case))
    state = 16 if case["bits"] == 32 else 4 + 4 / GROUP
    return {"bytes": n * ((4 if case["p16"] else 8) + (2 if case["g16"] else 4) + state + (2 if case["copy"] else 0)), "flops": 16 * n}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(st)
    if case["op"] == "lora":
        return _exact_lora(st)
    return _exact_adamw(st)


def _exact_norm(st):
    """Sample by sample; gradients by differentiating the definition."""
    c = st["case"]
    ys, stats, dxs, dscales, dshifts = [], [], [], [], []
    for i in range(0, c["M"], c["rows"]):
        rows, s = slice(i, min(c["M"], i + c["rows"])), i // c["rows"]
        x = st["x"][rows].double().requires_grad_(c["back"])
        scale = st["scale"][s].double().requires_grad_(c["back"])
        shift = (torch.zeros(c["K"], dtype=torch.float64, device=DEV) if st["shift"] is None else st["shift"][s].double()).requires_grad_(c["back"])
        var, mu = torch.var_mean(x, 1, correction=0)
        y = (x - mu[:, None]) / torch.sqrt(var + EPS)[:, None] * (scale + float(c["one"])) + shift
        if c["back"]:
            got = torch.autograd.grad(y, (x, scale, shift), st["dy"][rows].double())
            dxs.append(got[0]), dscales.append(got[1]), dshifts.append(got[2])
        else:
            ys.append(y), stats.append(torch.stack((mu, (var + EPS) ** -0.5), dim=1))
    if not c["back"]:
        return torch.cat(ys), torch.cat(stats)
    out = (torch.cat(dxs), torch.stack(dscales))
    return out + (torch.stack(dshifts),) if c["shift"] else out


def _exact_lora(st):
    """Request by request."""
    c = st["case"]
    n, r, K, N = c["n"], c["r"], c["K"], c["N"]
    if not c["back"]:
        y = st["y"].double()
    else:
        da = torch.zeros((n, r, K), dtype=torch.float64, device=DEV)
        db = torch.zeros((n, N, r), dtype=torch.float64, device=DEV)
        dx = st["dx"].double() if c["dx"] else None
    end = 0
    for length, i in zip(_ints(c["lens"]), _ints(c["ids"])):
        rows = slice(end, end + length)
        end += length
        if i < 0:
            continue
        x, a, b, s = st["x"][rows].double(), st["a"][i].double(), st["b"][i].double(), float(st["scaling"][i])
        if not c["back"]:
            y[rows] += x @ (s * (b @ a)).T
            continue
        dy, t = st["dy"][rows].double(), st["t"][rows, :r].double() + st["t"][rows, r:].double()
        da[i] += s * (b.T @ (dy.T @ x))
        db[i] += s * torch.einsum("mn,mr->nr", dy, t)
        if c["dx"]:
            dx[rows] += dy @ (s * (b @ a))
    return y if not c["back"] else (da, db, dx) if c["dx"] else (da, db)


def _exact_adamw(st):
    """Tensor by tensor.  What is held in 8 bits is rounded by chance and has no such value."""
    c = st["case"]
    eight, t = c["bits"] == 8, st["steps"] + 1
    p_out, m_out, v_out = st["p"].double(), None if eight else st["m"].double(), None if eight else st["v"].double()
    for first, size in zip(st["starts"], st["sizes"]):
        part = slice(first, first + size)
        g = st["g"][part].double()
        if eight:
            wide = slice(first, first + -(-size // GROUP) * GROUP)
            power = lambda s: torch.ldexp(torch.ones((), dtype=torch.float64, device=DEV), st[s][first // GROUP:][:-(-size // GROUP)].double() - 127.0)  # noqa: E731
            m = (st["m"][wide].view(torch.float8_e4m3fn).double().reshape(-1, GROUP) * power("ms")[:, None]).reshape(-1)[:size]
            v = (st["v"][wide].view(torch.float8_e5m2).double().reshape(-1, GROUP) * power("vs")[:, None]).reshape(-1)[:size]
        else:
            m, v = st["m"][part].double(), st["v"][part].double()
        m = torch.lerp(g, m, BETA1)
        v = torch.lerp(g ** 2, v, BETA2)
        if not eight:
            m_out[part], v_out[part] = m, v
        ahead = (m / (1.0 - BETA1 ** t)) / ((v / (1.0 - BETA2 ** t)) ** 0.5 + ADAM_EPS)
        p = p_out[part]
        p_out[part] = p - LR * DECAY * p - LR * ahead
    out = {"p": p_out, "m": m_out, "v": v_out}
    if eight:
        out["ms"] = out["vs"] = None
    if c["copy"]:
        copy = st["copy"].double()
        for first, size in zip(st["starts"], st["sizes"]):
            copy[first:first + size] = p_out[first:first + size]
        out["copy"] = copy
    return out
