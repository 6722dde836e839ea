"""Measured cases of the operators that stand between the quantized linears and the attention of a DiT block.

* 4-bit weight products (`nvfp4_matvec`, `mxfp4_matvec`): y = act(x) W^T + b for a few rows of BF16 x and a weight in
  NVFP4 or MXFP4 -- the modulation and embedding linears of a block, whose rows are samples and not tokens.
* Query / key preparation (`sol_qk_rotary`, `sol_qk_rotary_backward`): RMS norm of every head and rotary positions on
  the fused projection's q and k, and its gradients for the training phase.
* Block-sparse attention (`sol_select_blocks`, `sol_attention_blocks`): mean-pooled scores choose key blocks for each
  query block, and attention runs over the chosen blocks only.

Every operator has its plain form here (elementary torch operations in 32 bits, 64 where 32 would lose what matters)
and, with `own` true, the call a user makes.
"""
import math

import numpy as np
import torch

own = False


DEV = "cuda"
QBLOCK, KBLOCK = 256, 128


def _binding():
    from paper_2604_06916_b200 import binding as b
    return b


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one sample's modulation vector of a FLUX single-stream block: silu(c) W^T + b with three chunks of the width
        {"name": "matvec nvfp4 1x9216x3072", "op": "matvec", "fmt": "nv", "M": 1, "N": 9216, "K": 3072, "silu": True, "bias": True},
        # eight samples' modulation of a FLUX double-stream block: six chunks of the width
        {"name": "matvec nvfp4 8x18432x3072", "op": "matvec", "fmt": "nv", "M": 8, "N": 18432, "K": 3072, "silu": True, "bias": True},
        # an SD3.5 block's modulation for 24 samples (the images of one prompt that stage 2 renders), MXFP4
        {"name": "matvec mxfp4 24x14592x2432", "op": "matvec", "fmt": "mx", "M": 24, "N": 14592, "K": 2432, "silu": True, "bias": True},
        # q and k of one short text stream
        {"name": "rotary 1x333 text", "op": "rotary", "back": False, "B": 1, "S": 333, "H": 24, "Hk": 24, "D": 128, "axes": "16 56 56",
         "half": False, "norm": True, "far": 0, "scaling": "none"},
        # q and k of a FLUX block, eight samples at 1024 pixels: image rows and columns as positions, three axes
        {"name": "rotary 8x4608 flux", "op": "rotary", "back": False, "B": 8, "S": 4608, "H": 24, "Hk": 24, "D": 128, "axes": "16 56 56",
         "half": False, "norm": True, "far": 0, "scaling": "none"},
        # gradients of the same step for two samples, image and text tokens
        {"name": "rotary grad 2x4608 flux", "op": "rotary", "back": True, "B": 2, "S": 4608, "H": 24, "Hk": 24, "D": 128, "axes": "16 56 56",
         "half": False, "norm": True, "far": 0, "scaling": "none"},
        # half layout on part of the head, fewer key heads, far positions scaled for a long context
        {"name": "rotary grad 1x4099 half yarn", "op": "rotary", "back": True, "B": 1, "S": 4099, "H": 38, "Hk": 19, "D": 64, "axes": "32",
         "half": True, "norm": True, "far": 1000000, "scaling": "yarn"},
        # choosing a quarter of the key blocks of a FLUX block, two samples
        {"name": "select 2x4608", "op": "select", "B": 2, "S": 4608, "Skv": 4608, "H": 24, "Hk": 24, "D": 128, "count": 9, "first": 4, "lens": False},
        # a long token grid (a 2048-pixel image) with 64-wide heads and a ragged end
        {"name": "select 1x16421 d64", "op": "select", "B": 1, "S": 16421, "Skv": 16421, "H": 38, "Hk": 38, "D": 64, "count": 24, "first": 2, "lens": False},
        # a 512-pixel FLUX block: 1024 image and 512 text tokens, a third of the keys
        {"name": "attention 1x1536 of 4", "op": "attend", "B": 1, "S": 1536, "Skv": 1536, "H": 24, "Hk": 24, "D": 128, "count": 4, "first": 1, "lens": False},
        # two padded samples of a 64-wide model, ragged lengths
        {"name": "attention 2x4429 of 8 d64", "op": "attend", "B": 2, "S": 4429, "Skv": 4429, "H": 38, "Hk": 38, "D": 64, "count": 8, "first": 1, "lens": True},
        # four samples at 1024 pixels, a quarter of the keys
        {"name": "attention 4x4608 of 9", "op": "attend", "B": 4, "S": 4608, "Skv": 4608, "H": 24, "Hk": 24, "D": 128, "count": 9, "first": 4, "lens": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["matvec", "rotary", "rotary grad", "select", "attend"])
    if op == "matvec":
        K = 32 * _log(rng, 4, 480)
        N = 8 * _log(rng, 4, 2688)
        while N * K > 18432 * 3072:
            N = max(8, N // 16 * 8)
        return {"op": "matvec", "fmt": rng.choice(["nv", "mx"]), "M": _log(rng, 1, 64), "N": N, "K": K,
                "silu": rng.random() < 0.5, "bias": rng.random() < 0.7}
    if op.startswith("rotary"):
        D = rng.choice([32, 64, 128, 256])
        H = rng.randint(1, 40)
        Hk = rng.choice([h for h in range(1, H + 1) if H % h == 0])
        B = _log(rng, 1, 8)
        S = _log(rng, 1, 20000)
        while B * S * (H + Hk) * D > (8 if op == "rotary" else 2) * 4608 * 48 * 128:
            S = max(1, S // 2)
        rot = 8 * rng.randint(1, D // 8)
        axes = [rot]
        if rot >= 24 and rng.random() < 0.5:
            a = 2 * rng.randint(1, rot // 4)
            b = 2 * rng.randint(1, (rot - a) // 4)
            axes = [a, b, rot - a - b]
        one = len(axes) == 1 and axes[0] >= 8
        return {"op": "rotary", "back": op == "rotary grad", "B": B, "S": S, "H": H, "Hk": Hk, "D": D, "axes": " ".join(map(str, axes)), "half": rng.random() < 0.5,
                "norm": rng.random() < 0.7, "far": rng.choice([0, 0, 100000, 4000000]) if len(axes) == 1 else 0,
                "scaling": rng.choice(["none", "linear", "ntk", "yarn"]) if one else "none"}
    D = rng.choice([64, 128])
    H = rng.randint(1, 38)
    Hk = rng.choice([h for h in range(1, H + 1) if H % h == 0])
    B = _log(rng, 1, 4)
    S = _log(rng, 1, 16000)
    Skv = S if rng.random() < 0.7 else _log(rng, 1, 16000)
    if op == "select":
        while B * (S * H + Skv * Hk) * D > 1 * 16421 * 76 * 64:
            S, Skv = max(1, S // 2), max(1, Skv // 2)
    nk = -(-Skv // KBLOCK)
    count = rng.randint(1, min(nk, 24))
    first = rng.randint(0, min(2, count))
    if op == "attend":
        while B * H * D * -(-S // QBLOCK) * count > 4 * 24 * 128 * 18 * 9:
            S, count = max(1, S // 2), max(1, count // 2)
            first = min(first, count)
    return {"op": op, "B": B, "S": S, "Skv": Skv, "H": H, "Hk": Hk, "D": D, "count": count, "first": first, "lens": rng.random() < 0.4}


def _axes(case):
    """Rotated columns of each position axis."""
    return [int(d) for d in case["axes"].split()]


# ------------------------------------------------------------------------------------------------ inputs
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _scale_offsets(N, blocks, device):
    """Byte offsets [N, blocks] of the block scales in the 512-byte chunks of 128 rows x 4 blocks that the linears use."""
    r = torch.arange(N, device=device)[:, None]
    b = torch.arange(blocks, device=device)[None, :]
    return ((r // 128) * -(-blocks // 4) + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4


def _weights(fmt, N, K, g):
    """A normal weight of deviation K^-1/2, quantized block by block: nibbles, chunked scales, tensor scale."""
    w = torch.randn((N, K), generator=g, device=DEV) * K ** -0.5
    size = 16 if fmt == "nv" else 32
    blk = w.reshape(N, K // size, size)
    amax = blk.abs().amax(2)
    if fmt == "nv":
        T = (amax.max() / 2688.0).reshape(1)
        code = (amax / (6.0 * T)).to(torch.float8_e4m3fn)
        real = code.float() * T
        code = code.view(torch.uint8)
    else:
        T = None
        e = torch.floor(torch.log2(amax)) - 2.0
        real = torch.exp2(e)
        code = (e + 127.0).to(torch.uint8)
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEV)
    v = blk / real[:, :, None]
    nib = torch.bucketize(v.abs(), edges).to(torch.uint8) | ((v < 0).to(torch.uint8) << 3)
    nib = nib.reshape(N, K // 2, 2)
    q = (nib[:, :, 0] | (nib[:, :, 1] << 4)).contiguous()
    sf = torch.zeros(-(-N // 128) * -(-(K // size) // 4) * 512, dtype=torch.uint8, device=DEV)
    sf[_scale_offsets(N, K // size, DEV)] = code
    return q, sf, T


def _frequencies(case):
    """Radians per position of each rotated pair, and the factor on cosine and sine (64 bits)."""
    theta, scale, out = 10000.0, 1.0, []
    for d in _axes(case):
        i = torch.arange(d // 2, dtype=torch.float64)
        factor = 8.0
        base = theta * factor ** (d / (d - 2.0)) if case["scaling"] == "ntk" and d > 2 else theta
        f = base ** (-2.0 * i / d)
        if case["scaling"] == "linear":
            f = f / factor
        if case["scaling"] == "yarn":
            turn = lambda beta: d * math.log(4096.0 / (beta * 2.0 * math.pi)) / (2.0 * math.log(theta))  # noqa: E731
            lo, hi = max(math.floor(turn(32.0)), 0), min(math.ceil(turn(1.0)), d - 1)
            ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
            f = f / factor * ramp + f * (1.0 - ramp)
            scale = 0.1 * math.log(factor) + 1.0
        out.append(f)
    return torch.cat(out).to(DEV), scale


def _positions(case, g):
    S, axes = case["S"], len(_axes(case))
    if axes == 1:
        return case["far"] + torch.arange(S, device=DEV)[:, None]
    # text tokens at the origin, then an image grid in row order
    text = min(512, S // 3)
    side = max(1, math.isqrt(S - text))
    n = torch.arange(S - text, device=DEV)
    ids = torch.zeros((S, axes), dtype=torch.int64, device=DEV)
    ids[text:, 1], ids[text:, 2] = n // side, n % side
    return ids


def _tokens(B, S, H, D, g, field):
    """Normal tokens with a part that changes slowly along the sequence, as neighbouring patches share theirs."""
    x = torch.randn((B, S, H * D), generator=g, device=DEV)
    if field:
        slow = torch.randn((B, -(-S // 64), H * D), generator=g, device=DEV)
        x += 0.7 * slow.repeat_interleave(64, dim=1)[:, :S]
    return x.to(torch.bfloat16)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 13)
    st = {"case": case}
    if case["op"] == "matvec":
        st["x"] = (1.5 * torch.randn((case["M"], case["K"]), generator=g, device=DEV)).to(torch.bfloat16)
        st["wq"], st["wsf"], st["wts"] = _weights(case["fmt"], case["N"], case["K"], g)
        st["bias"] = (0.1 * torch.randn(case["N"], generator=g, device=DEV)).to(torch.bfloat16) if case["bias"] else None
        return st
    B, S, H, Hk, D = case["B"], case["S"], case["H"], case["Hk"], case["D"]
    if case["op"] == "rotary":
        # q and k are column slices of one fused projection output (q, k, v side by side)
        fused = _tokens(B, S, H + 2 * Hk, D, g, False)
        st["q"] = fused[:, :, :H * D].unflatten(2, (H, D))
        st["k"] = fused[:, :, H * D:(H + Hk) * D].unflatten(2, (Hk, D))
        st["qw"] = st["kw"] = None
        if case["norm"]:
            st["qw"] = (1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(torch.bfloat16)
            st["kw"] = (1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(torch.bfloat16)
        st["axes"] = _axes(case)
        st["freqs"], st["scale"] = _frequencies(case)
        st["pos"] = _positions(case, g)
        if case["back"]:
            st["dq"] = _tokens(B, S, H, D, g, False).unflatten(2, (H, D))
            st["dk"] = _tokens(B, S, Hk, D, g, False).unflatten(2, (Hk, D))
        return st
    Skv, nq, nk = case["Skv"], -(-S // QBLOCK), -(-case["Skv"] // KBLOCK)
    st["q"] = _tokens(B, S, H, D, g, True).unflatten(2, (H, D))
    st["k"] = _tokens(B, Skv, Hk, D, g, True).unflatten(2, (Hk, D))
    st["lens"] = torch.randint(max(1, Skv // 2), Skv + 1, (B,), generator=g, device=DEV).to(torch.int32) if case["lens"] else None
    if case["op"] == "attend":
        st["v"] = (0.5 * _tokens(B, Skv, Hk, D, g, False).float()).to(torch.bfloat16).unflatten(2, (Hk, D))
        # a list as a selection leaves it: the first blocks always, the others anywhere, ascending, -1 behind the last
        left = nk if st["lens"] is None else ((st["lens"].long() + KBLOCK - 1) // KBLOCK).reshape(B, 1, 1, 1)
        score = torch.rand((B, H, nq, nk), generator=g, device=DEV)
        at = torch.arange(nk, device=DEV)
        score = torch.where(at < case["first"], 2.0 + score, score)
        score = torch.where(at < left, score, torch.full_like(score, -1.0))
        top, idx = score.topk(case["count"], dim=3)
        idx = torch.where(top >= 0, idx, nk).sort(dim=3).values
        st["counts"] = (idx < nk).sum(3).to(torch.int32)
        st["blocks"] = torch.where(idx < nk, idx, -1).to(torch.int32).contiguous()
    return st


# ------------------------------------------------------------------------------------------------ the calls
def run(st):
    c = st["case"]
    if c["op"] == "matvec":
        return _own_matvec(st) if own else _plain_matvec(st)
    if c["op"] == "rotary":
        if own:
            return _own_rotary(st)
        return _plain_rotary_grad(st) if c["back"] else _plain_rotary(st)
    if c["op"] == "select":
        return _own_select(st) if own else _plain_select(st)
    return _own_attend(st) if own else _plain_attend(st)


def _own_matvec(st):
    b, c = _binding(), st["case"]
    act = b.ACT_SILU if c["silu"] else b.ACT_NONE
    if c["fmt"] == "nv":
        return b.nvfp4_matvec(st["x"], st["wq"], st["wsf"], st["wts"], st["bias"], activation=act)
    return b.mxfp4_matvec(st["x"], st["wq"], st["wsf"], st["bias"], activation=act)


def _own_rotary(st):
    b, c = _binding(), st["case"]
    layout = b.ROTARY_HALF if c["half"] else b.ROTARY_INTERLEAVED
    kw = dict(axis_dims=st["axes"], layout=layout, q_weight=st["qw"], k_weight=st["kw"], scale=st["scale"])
    if c["back"]:
        got = b.sol_qk_rotary_backward(st["dq"], st["dk"], st["q"], st["k"], st["pos"], st["freqs"], **kw)
        return [t for t in got if t is not None]
    return b.sol_qk_rotary(st["q"], st["k"], st["pos"], st["freqs"], **kw)


def _own_select(st):
    c = st["case"]
    return _binding().sol_select_blocks(st["q"], st["k"], c["count"], keep_first=c["first"], kv_lens=st["lens"], with_scores=True)


def _own_attend(st):
    return _binding().sol_attention_blocks(st["q"], st["k"], st["v"], st["blocks"], st["counts"], kv_lens=st["lens"])


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_matvec(st):
    x, q, c = st["x"].float(), st["wq"], st["case"]
    N, K, size = c["N"], c["K"], 16 if c["fmt"] == "nv" else 32
    lut = torch.tensor(E2M1, device=q.device)
    w = torch.stack((lut[(q & 15).int()], lut[(q >> 4).int()]), dim=2).reshape(N, K // size, size)
    code = st["wsf"][_scale_offsets(N, K // size, q.device)]
    if c["fmt"] == "nv":
        e, m = (code >> 3).float(), (code & 7).float()
        s = torch.where(e > 0, (1.0 + m / 8.0) * torch.exp2(e - 7.0), m / 512.0) * st["wts"]
    else:
        s = torch.exp2(code.float() - 127.0)
    w = (w * s[:, :, None]).reshape(N, K)
    if c["silu"]:
        x = x / (1.0 + torch.exp(-x))
    y = x @ w.t()
    if st["bias"] is not None:
        y = y + st["bias"].float()
    return y.to(torch.bfloat16)


def _cos_sin(st):
    """[S, 1, pairs] cosine and sine: the angles of far positions are formed and reduced in 64 bits."""
    axis = torch.repeat_interleave(torch.arange(len(st["axes"])), torch.tensor(st["axes"]) // 2).to(DEV)
    a = st["pos"][:, axis].double() * st["freqs"]
    return (st["scale"] * torch.cos(a)).float()[:, None], (st["scale"] * torch.sin(a)).float()[:, None]


def _pairs(x, half):
    """The two members of each rotated pair of the leading columns."""
    if half:
        h = x.shape[-1] // 2
        return x[..., :h], x[..., h:]
    return x[..., 0::2], x[..., 1::2]


def _join(a, b, half):
    return torch.cat((a, b), dim=-1) if half else torch.stack((a, b), dim=-1).flatten(-2)


def _plain_rotary(st):
    c, rot = st["case"], sum(st["axes"])
    cos, sin = _cos_sin(st)
    out = []
    for x, w in ((st["q"], st["qw"]), (st["k"], st["kw"])):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(3, keepdim=True) + 1e-6) * w.float()
        a, b = _pairs(x[..., :rot], c["half"])
        y = _join(a * cos - b * sin, b * cos + a * sin, c["half"])
        out.append(torch.cat((y, x[..., rot:]), dim=3).to(torch.bfloat16))
    return tuple(out)


def _plain_rotary_grad(st):
    c, rot = st["case"], sum(st["axes"])
    cos, sin = _cos_sin(st)
    grads, weights = [], []
    for x, w, dy in ((st["q"], st["qw"], st["dq"]), (st["k"], st["kw"], st["dk"])):
        x, dy = x.float(), dy.float()
        a, b = _pairs(dy[..., :rot], c["half"])
        dn = torch.cat((_join(a * cos + b * sin, b * cos - a * sin, c["half"]), dy[..., rot:]), dim=3)
        if w is None:
            grads.append(dn.to(torch.bfloat16))
            continue
        r = torch.rsqrt(x.square().mean(3, keepdim=True) + 1e-6)
        xhat = x * r
        dh = dn * w.float()
        grads.append((r * (dh - xhat * (dh * xhat).mean(3, keepdim=True))).to(torch.bfloat16))
        weights.append((dn * xhat).sum((0, 1, 2), dtype=torch.float64).float())
    return grads + weights


def _pooled(x, size, lens):
    """[B, H, blocks, D] means of the rows that exist (64 bits: the choice of a block must not hang on a rounding), and how many exist."""
    B, S, H, D = x.shape
    n = -(-S // size)
    x = x.double()
    if lens is not None:
        x = torch.where(torch.arange(S, device=x.device)[None, :, None, None] < lens.long()[:, None, None, None], x, 0.0)
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, n * size - S)).reshape(B, n, size, H, D).sum(2)
    length = torch.full((B,), S, device=x.device) if lens is None else lens.long().clamp(0, S)
    rows = (length[:, None] - size * torch.arange(n, device=x.device)).clamp(0, size)
    return (x / rows.clamp(min=1)[:, :, None, None]).permute(0, 2, 1, 3), rows


def _plain_select(st):
    c = st["case"]
    H, Hk, count = c["H"], c["Hk"], c["count"]
    pq, _ = _pooled(st["q"], QBLOCK, None)
    pk, rows = _pooled(st["k"], KBLOCK, st["lens"])
    pk = pk.repeat_interleave(H // Hk, dim=1)
    score = pq @ pk.transpose(2, 3)
    nk = score.shape[3]
    at = torch.arange(nk, device=score.device)
    score = torch.where((rows > 0)[:, None, None, :], score, -math.inf)
    rank = torch.where((at < c["first"]) & (rows > 0)[:, None, None, :], math.inf, score)
    order = torch.sort(rank, dim=3, descending=True, stable=True)
    idx = torch.where(order.values > -math.inf, order.indices, nk)[..., :count]
    idx = idx.sort(dim=3).values
    live = idx < nk
    chosen = torch.where(live, torch.gather(score, 3, idx.clamp(max=nk - 1)), -math.inf)
    return torch.where(live, idx, -1).to(torch.int32), live.sum(3).to(torch.int32), chosen.float()


def _plain_attend(st):
    """Gathers the listed blocks of every query block and runs the softmax over them."""
    c = st["case"]
    B, S, Skv, H, Hk, D, count = c["B"], c["S"], c["Skv"], c["H"], c["Hk"], c["D"], c["count"]
    nq, nk = -(-S // QBLOCK), -(-Skv // KBLOCK)
    pad = lambda x, n, size: torch.nn.functional.pad(x.float(), (0, 0, 0, 0, 0, n * size - x.shape[1])).reshape(B, n, size, -1, D).permute(0, 3, 1, 2, 4)  # noqa: E731
    q, k, v = pad(st["q"], nq, QBLOCK), pad(st["k"], nk, KBLOCK), pad(st["v"], nk, KBLOCK)
    at = st["blocks"].long().clamp(min=0)
    b = torch.arange(B, device=at.device)[:, None, None, None]
    h = (torch.arange(H, device=at.device) // (H // Hk))[None, :, None, None]
    k, v = (t[b, h, at].reshape(B, H, nq, count * KBLOCK, D) for t in (k, v))
    key = at[..., None] * KBLOCK + torch.arange(KBLOCK, device=at.device)
    length = torch.full((B,), Skv, device=at.device) if st["lens"] is None else st["lens"].long()
    live = (torch.arange(count, device=at.device) < st["counts"][..., None])[..., None] & (key < length[:, None, None, None, None])
    live = live.reshape(B, H, nq, 1, count * KBLOCK)
    s = q @ k.transpose(3, 4) * D ** -0.5
    s = torch.where(live, s, -math.inf)
    p = torch.exp(s - s.amax(4, keepdim=True).clamp(min=-1e30))
    p = torch.where(live, p, 0.0)
    o = (p @ v) / p.sum(4, keepdim=True).clamp(min=1e-30)
    return o.permute(0, 2, 3, 1, 4).reshape(B, nq * QBLOCK, H, D)[:, :S].to(torch.bfloat16).contiguous()


# ------------------------------------------------------------------------------------------------ work
def work(case):
    if case["op"] == "matvec":
        M, N, K = case["M"], case["N"], case["K"]
        size = 16 if case["fmt"] == "nv" else 32
        return {"bytes": N * K // 2 + N * K // size + 2 * M * K + 2 * M * N + 2 * N, "flops": 2 * M * N * K}
    B, S, H, Hk, D = case["B"], case["S"], case["H"], case["Hk"], case["D"]
    if case["op"] == "rotary":
        el = B * S * (H + Hk) * D
        return {"bytes": el * 2 * (3 if case["back"] else 2) + S * len(_axes(case)) * 8, "flops": el * (16 if case["back"] else 8)}
    Skv, count = case["Skv"], case["count"]
    nq, nk = -(-S // QBLOCK), -(-Skv // KBLOCK)
    if case["op"] == "select":
        return {"bytes": 2 * D * B * (S * H + Skv * Hk) + 4 * B * H * nq * (2 * count + 1), "flops": D * B * (S * H + Skv * Hk) + 2 * B * H * nq * nk * D}
    pairs = B * H * S * min(count * KBLOCK, Skv)
    return {"bytes": 2 * D * B * (2 * S * H + 2 * Skv * Hk) + 4 * B * H * nq * (count + 1), "flops": 4 * pairs * D}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    with torch.no_grad():
        if case["op"] == "matvec":
            return _exact_matvec(st)
    if case["op"] == "rotary":
        return _exact_rotary(st)
    with torch.no_grad():
        return _exact_select(st) if case["op"] == "select" else _exact_attend(st)


def _exact_matvec(st):
    """Codes taken apart bit by bit: (-1)^s 2^(e-1) (1 + m/2), or m/2 for e = 0."""
    c, out = st["case"], []
    size = 16 if c["fmt"] == "nv" else 32
    x = st["x"].double()
    if c["silu"]:
        x = x * torch.sigmoid(x)
    for n0 in range(0, c["N"], 4096):
        n1 = min(c["N"], n0 + 4096)
        q = st["wq"][n0:n1].to(torch.int32)
        n = torch.empty((n1 - n0, c["K"]), dtype=torch.int32, device=q.device)
        n[:, 0::2], n[:, 1::2] = q % 16, q // 16
        e, m = n // 2 % 4, (n % 2).double()
        w = torch.where(e == 0, m / 2, torch.ldexp(1 + m / 2, e - 1)) * (1 - 2 * (n // 8)).double()
        row, blk = np.meshgrid(np.arange(n0, n1), np.arange(c["K"] // size), indexing="ij")
        chunk = row // 128 * ((c["K"] // size + 3) // 4) + blk // 4
        at = torch.from_numpy(chunk * 512 + row % 32 * 16 + row // 32 % 4 * 4 + blk % 4).to(q.device)
        code = st["wsf"][at].to(torch.int32)
        if c["fmt"] == "nv":
            s = code.to(torch.uint8).view(torch.float8_e4m3fn).double() * st["wts"].double()
        else:
            s = torch.ldexp(torch.ones_like(code, dtype=torch.float64), code - 127)
        w *= torch.repeat_interleave(s, size, dim=1)
        out.append(torch.einsum("mk,nk->mn", x, w))
    y = torch.cat(out, dim=1)
    return y if st["bias"] is None else y + st["bias"].double()


def _exact_rotary(st):
    """Pairs as complex numbers turned by exp(i angle); gradients by differentiating that in 64 bits."""
    c = st["case"]
    rot, parts = sum(st["axes"]), []
    first = 0
    for n, d in enumerate(st["axes"]):
        parts.append(torch.outer(st["pos"][:, n].double(), st["freqs"][first:first + d // 2]))
        first += d // 2
    turn = torch.polar(torch.full_like(torch.cat(parts, 1), st["scale"]), torch.cat(parts, 1))[None, :, None]
    values, weights = [], []
    for x, w, dy in ((st["q"], st["qw"], st.get("dq")), (st["k"], st["kw"], st.get("dk"))):
        x = x.double().requires_grad_(c["back"])
        h = x
        if w is not None:
            w = w.double().requires_grad_(c["back"])
            h = torch.sqrt(1.0 / ((x * x).sum(3, keepdim=True) / c["D"] + 1e-6)) * x * w
        head, rest = h[..., :rot], h[..., rot:]
        z = head.unflatten(3, (2, rot // 2)).transpose(3, 4) if c["half"] else head.unflatten(3, (rot // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        z = (z.transpose(3, 4) if c["half"] else z).flatten(3)
        y = torch.cat((z, rest), dim=3)
        if not c["back"]:
            values.append(y)
            continue
        got = torch.autograd.grad((y * dy.double()).sum(), [x] + ([w] if w is not None else []))
        values.append(got[0])
        weights += list(got[1:])
    return values + weights if c["back"] else tuple(values)


def _exact_select(st):
    """Means by products with averaging matrices; every row of scores ordered by itself, lower blocks first among equals."""
    c = st["case"]
    B, S, Skv, H, Hk = c["B"], c["S"], c["Skv"], c["H"], c["Hk"]
    lens = [Skv] * B if st["lens"] is None else st["lens"].tolist()
    blocks = np.full((B, H, -(-S // QBLOCK), c["count"]), -1, dtype=np.int32)
    counts = np.zeros(blocks.shape[:3], dtype=np.int32)
    chosen = np.full(blocks.shape, -np.inf)

    def averaging(length, size):
        at = torch.arange(length, device=DEV)
        m = (at // size == torch.arange(-(-length // size), device=DEV)[:, None]).double()
        return m / m.sum(1, keepdim=True)

    aq = averaging(S, QBLOCK)
    for i in range(B):
        ak = averaging(lens[i], KBLOCK)
        nk = ak.shape[0]
        for h in range(H):
            mq, mk = aq @ st["q"][i, :, h].double(), ak @ st["k"][i, :lens[i], h * Hk // H].double()
            score = torch.einsum("nd,md->nm", mq, mk).cpu().numpy()
            rank = score.copy()
            rank[:, :c["first"]] = np.inf
            got = np.sort(np.argsort(-rank, axis=1, kind="stable")[:, :c["count"]], axis=1)
            blocks[i, h, :, :got.shape[1]] = got
            chosen[i, h, :, :got.shape[1]] = np.take_along_axis(score, got, axis=1)
            counts[i, h] = min(nk, c["count"])
    return torch.from_numpy(blocks), torch.from_numpy(counts), torch.from_numpy(chosen)


def _exact_attend(st):
    """Row block by row block, over the keys that the list names."""
    c = st["case"]
    B, S, Skv, H, Hk, D = c["B"], c["S"], c["Skv"], c["H"], c["Hk"], c["D"]
    blocks, counts = st["blocks"].cpu().numpy(), st["counts"].cpu().numpy()
    lens = [Skv] * B if st["lens"] is None else st["lens"].tolist()
    if blocks.shape[0] * blocks.shape[1] * blocks.shape[2] > 6000:
        return None
    out = torch.zeros((B, S, H, D), dtype=torch.float64, device=DEV)
    q, k, v = (st[n].double() for n in "qkv")
    step = np.arange(KBLOCK)
    for i in range(B):
        for h in range(H):
            for n in range(blocks.shape[2]):
                keys = (blocks[i, h, n, :counts[i, h, n], None].astype(np.int64) * KBLOCK + step).reshape(-1)
                keys = torch.from_numpy(keys[keys < lens[i]]).to(DEV)
                if keys.numel():
                    rows = slice(n * QBLOCK, min(S, (n + 1) * QBLOCK))
                    p = torch.softmax(torch.einsum("sd,td->st", q[i, rows, h], k[i, keys, h * Hk // H]) / math.sqrt(D), dim=1)
                    out[i, rows, h] = p @ v[i, keys, h * Hk // H]
    return out
