"""What is measured of the operators around the layer in its transformer block: the cast of activations and weights to 8-bit
floating point with a scale for each block of 128 (`quantize`), the projections as products of such operands (`scaled_matmul`) and
attention to an encoder's states (`cross_attention`).

`run` computes them in elementary torch operations, or, where `own` is set, through the library's binding.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
BLOCK = 128


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the 768p-shaped clip's read-outs (86 frames of 4080 tokens, 40 heads of 128) on their way to the output projection
        dict(name="quantize 768p", op="quantize", dtype="bf16", rows=350880, cols=5120, tile=1),
        # a projection's weights when a model is loaded, in square blocks; ragged in both directions, 32 bits
        dict(name="quantize weights f32", op="quantize", dtype="f32", rows=5000, cols=2600, tile=128),
        # one token through a projection: latency, and the weights' bytes
        dict(name="project one", op="project", dtype="bf16", m=1, n=5120, k=5120, bias=True, add=False, pow2=False),
        # one token of each request of a serving batch
        dict(name="project batch 48", op="project", dtype="bf16", m=48, n=5120, k=5120, bias=False, add=True, pow2=False),
        # a short prompt, 32-bit results, a last block of 72 channels, an odd number of features
        dict(name="project f32 prompt 77", op="project", dtype="f32", m=77, n=1001, k=1352, bias=True, add=False, pow2=True),
        # the 480p-shaped clip's output projection added to the other branch's
        dict(name="project 480p", op="project", dtype="bf16", m=32760, n=1024, k=1024, bias=False, add=True, pow2=True),
        # half of the 768p-shaped clip
        dict(name="project 768p", op="project", dtype="bf16", m=175440, n=5120, k=5120, bias=True, add=False, pow2=False),
        # the tiny configuration's tokens against a masked prompt, 32 bits: latency
        dict(name="cross f32 tiny", op="cross", dtype="f32", d=64, heads=2, key_heads=2, batch=1, queries=256, keys=77,
             packed=False, ragged=False, masked=True),
        # one token of each of 32 requests, each against its own encoder states (audio, images), packed
        dict(name="cross step 32", op="cross", dtype="bf16", d=128, heads=32, key_heads=8, batch=32, queries=1, keys=1500,
             packed=True, ragged=True, masked=False),
        # the 480p-shaped clip, guided and unguided, against two short prompts of a padded batch
        dict(name="cross 480p", op="cross", dtype="bf16", d=128, heads=8, key_heads=8, batch=2, queries=32760, keys=77,
             packed=False, ragged=True, masked=False),
        # a quarter of the 768p-shaped clip against a long prompt, 40 heads
        dict(name="cross 768p", op="cross", dtype="bf16", d=128, heads=40, key_heads=40, batch=1, queries=87720, keys=512,
             packed=False, ragged=False, masked=False),
        # one frame against the states of a whole clip, some of them masked, two query heads to a key head
        dict(name="cross frame to clip", op="cross", dtype="bf16", d=64, heads=8, key_heads=4, batch=1, queries=1560, keys=32760,
             packed=False, ragged=False, masked=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("quantize", "project", "project", "cross", "cross", "cross"))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if op == "quantize":
        cols = _log_int(rng, 64, 12000)
        return dict(op=op, dtype=dtype, rows=_log_int(rng, 1, min(300000, 10 ** 9 // cols)), cols=cols,
                    tile=rng.choice((1, 1, 128)))
    if op == "project":
        n, k = _log_int(rng, 64, 9000), _log_int(rng, 64, 9000)
        return dict(op=op, dtype=dtype, m=_log_int(rng, 1, min(150000, 4 * 10 ** 12 // (n * k))), n=n, k=k, bias=rng.random() < 0.5,
                    add=rng.random() < 0.5, pow2=rng.random() < 0.5)
    key_heads = rng.choice((1, 2, 3, 4, 8, 12, 40))
    heads = key_heads * rng.choice((1, 1, 2, 3, 8))
    d = 64 if rng.random() < 0.3 else 128
    keys = _log_int(rng, 1, 20000)
    batch = _log_int(rng, 1, max(1, min(64, 2 ** 26 // (keys * key_heads * d))))
    most = (2 ** 29 if dtype == "bf16" else 2 ** 27) // (heads * keys * batch)
    return dict(op=op, dtype=dtype, d=d, heads=heads, key_heads=key_heads, batch=batch, queries=_log_int(rng, 1, max(1, min(60000, most))),
                keys=keys, packed=rng.random() < 0.4, ragged=rng.random() < 0.6, masked=rng.random() < 0.3)


def _lengths(case):
    """Keys of each batch row: all of them the same, or anything from one to the longest."""
    if not case["ragged"]:
        return [case["keys"]] * case["batch"]
    r = random.Random(case["keys"] * 1000 + case["batch"])
    return [case["keys"] if i == 0 else r.randint(1, case["keys"]) for i in range(case["batch"])]


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _scale_of(blocks, pow2):
    """Scales of blocks (the last dimension) with the largest magnitude at 448, or within a factor of two of it."""
    s = blocks.abs().amax(-1) / 448.0
    return torch.exp2(torch.ceil(torch.log2(s))) if pow2 else s


def _weights(gen, n, k, pow2):
    """A projection's weights as a checkpoint has them: 8 bits [n, k], a scale for each square block."""
    nb, kb = -(-n // BLOCK), -(-k // BLOCK)
    spread = torch.exp(0.3 * torch.randn(n, 1, generator=gen, device=DEV))
    w = torch.zeros(nb * BLOCK, kb * BLOCK, device=DEV)
    w[:n, :k] = torch.randn(n, k, generator=gen, device=DEV) * spread / math.sqrt(k)
    w = w.view(nb, BLOCK, kb, BLOCK).transpose(1, 2)
    s = _scale_of(w.flatten(2), pow2)
    w = (w / s[..., None, None]).to(torch.float8_e4m3fn).transpose(1, 2).reshape(nb * BLOCK, kb * BLOCK)
    rows = -(-k // 16) * 16                                                  # rows begin at multiples of 16 bytes
    room = torch.empty(n, rows, device=DEV, dtype=torch.float8_e4m3fn)
    room[:, :k] = w[:n, :k]
    return room[:, :k], s


def _activations(gen, rows, cols, dt):
    """Tokens whose sizes differ, with a few channels far larger than the rest."""
    loud = 1 + 20.0 * (torch.rand(cols, generator=gen, device=DEV) < 0.01).to(dt)
    size = torch.exp(0.5 * torch.randn(rows, 1, generator=gen, device=DEV)).to(dt)
    return torch.randn(rows, cols, generator=gen, device=DEV, dtype=dt).mul_(loud).mul_(size)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt = _dtype(case)
    s = dict(case=case)
    if case["op"] == "quantize":
        s["x"] = _activations(gen, case["rows"], case["cols"], dt)
    elif case["op"] == "project":
        s["x"] = _activations(gen, case["m"], case["k"], dt)
        s["w"], s["w_scale"] = _weights(gen, case["n"], case["k"], case["pow2"])
        s["bias"] = torch.randn(case["n"], generator=gen, device=DEV) if case["bias"] else None
        s["add"] = torch.randn(case["m"], case["n"], generator=gen, device=DEV, dtype=dt) if case["add"] else None
    else:
        h, hk, d, b = case["heads"], case["key_heads"], case["d"], case["batch"]
        lens = _lengths(case)
        n = sum(lens) if case["packed"] else b * case["keys"]
        lead = (n,) if case["packed"] else (b, case["keys"])
        s["q"] = torch.randn(b, case["queries"], h, d, generator=gen, device=DEV, dtype=dt)
        s["k"] = (1.5 * torch.randn(*lead, hk, d, generator=gen, device=DEV)).to(dt)
        s["v"] = torch.randn(*lead, hk, d, generator=gen, device=DEV, dtype=dt)
        s["cu_seqlens"] = torch.tensor([0] + lens).cumsum(0).to(torch.int32).to(DEV) if case["packed"] else None
        s["lengths"] = torch.tensor(lens, dtype=torch.int32, device=DEV) if case["ragged"] and not case["packed"] else None
        s["mask"] = torch.rand(*lead, generator=gen, device=DEV) < 0.8 if case["masked"] else None
        s["scale"] = d ** -0.5
    if own:
        from paper_2609_20744_b200 import binding
        s["vda"] = binding.Vda(case.get("d", 128), case["dtype"])
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return {"quantize": _quantize_case, "project": _project, "cross": _cross}[op](s)


def _own(s, op):
    if op == "quantize":
        x8, scale = s["vda"].quantize(s["x"], rows=s["case"]["tile"])
        return {"x8": x8, "scale": scale}
    if op == "project":
        x8, scale = s["vda"].quantize(s["x"])
        return s["vda"].scaled_matmul(x8, scale, s["w"], s["w_scale"], bias=s["bias"], add=s["add"])
    out, lse = s["vda"].cross_attention(s["q"], s["k"], s["v"], cu_seqlens=s["cu_seqlens"], lengths=s["lengths"], mask=s["mask"],
                                        scale=s["scale"], lse=True)
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------------------------------------ plain forms
def _blocks(x, tile):
    """x [rows, cols] as [row blocks, column blocks, tile, 128], zeros behind its ends."""
    r, c = x.shape
    rb, cb = -(-r // tile), -(-c // BLOCK)
    if (rb * tile, cb * BLOCK) != (r, c):
        room = torch.zeros(rb * tile, cb * BLOCK, device=x.device, dtype=x.dtype)
        room[:r, :c] = x
        x = room
    return x.view(rb, tile, cb, BLOCK).transpose(1, 2)


def _quantize(x, tile):
    """The smallest power of two that brings a block's largest magnitude to 448 or less (1 for a block of zeros), and the block
    divided by it, rounded to 8 bits."""
    r, c = x.shape
    b = _blocks(x.float(), tile)
    mantissa, exponent = torch.frexp(b.abs().amax((-2, -1)))
    scale = torch.ldexp(torch.ones_like(mantissa), exponent - 9 + (mantissa > 0.875).int())
    scale = torch.where(mantissa > 0, scale, 1.0)
    b = (b / scale[..., None, None]).to(torch.float8_e4m3fn)
    return b.transpose(1, 2).reshape(b.shape[0] * tile, -1)[:r, :c], scale


def _quantize_case(s):
    x8, scale = _quantize(s["x"], s["case"]["tile"])
    return {"x8": x8, "scale": scale}


def _project(s):
    x8, scale = _quantize(s["x"], 1)
    m, k = x8.shape
    n = s["w"].shape[0]
    x = (_blocks(x8.float(), 1) * scale[..., None, None]).reshape(m, -1)
    w = (_blocks(s["w"].float(), BLOCK) * s["w_scale"][..., None, None]).transpose(1, 2).reshape(-1, x.shape[1])[:n]
    out = x @ w.mT
    if s["bias"] is not None:
        out += s["bias"]
    if s["add"] is not None:
        out += s["add"]
    return out.to(_dtype(s["case"]))


def _padded(s):
    """k, v [batch, keys, key_heads, d] in 32 bits and which keys count [batch, keys]."""
    c = s["case"]
    k, v, mask = s["k"].float(), s["v"].float(), s["mask"]
    at = torch.arange(c["keys"], device=DEV)
    if s["cu_seqlens"] is not None:
        first = s["cu_seqlens"][:-1].long()
        there = at[None] < (s["cu_seqlens"][1:].long() - first)[:, None]
        row = (first[:, None] + at[None]).clamp(max=k.shape[0] - 1)
        k, v = k[row], v[row]
        return k, v, there if mask is None else there & mask[row]
    there = at[None] < s["lengths"][:, None] if s["lengths"] is not None else torch.ones(c["batch"], c["keys"], device=DEV, dtype=torch.bool)
    return k, v, there if mask is None else there & mask


def _cross(s):
    c = s["case"]
    b, lq, h, hk, d = c["batch"], c["queries"], c["heads"], c["key_heads"], c["d"]
    k, v, there = _padded(s)
    q = s["q"].float().view(b, lq, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d)
    p = (q * s["scale"]) @ k.permute(0, 2, 3, 1)                             # [b, hk, group x queries, keys]
    p.masked_fill_(~there[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    total = p.sub_(top).exp_().sum(-1, keepdim=True)
    out = p @ v.transpose(1, 2) / torch.where(total > 0, total, 1.0)
    lse = torch.log(total) + top
    back = lambda x: x.view(b, hk, h // hk, lq, -1).permute(0, 3, 1, 2, 4).reshape(b, lq, h, -1)  # noqa: E731
    return {"out": back(out).to(_dtype(c)), "lse": back(lse)[..., 0]}


# ------------------------------------------------------------------------------------------------ floors
def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "quantize":
        r, c, t = case["rows"], case["cols"], case["tile"]
        return {"bytes": r * c * (e + 1) + 4 * -(-r // t) * -(-c // BLOCK), "flops": 3 * r * c}
    if case["op"] == "project":
        m, n, k = case["m"], case["n"], case["k"]
        blocks = -(-n // BLOCK) * -(-k // BLOCK)
        return {"bytes": m * k * e + n * k + 4 * blocks + m * n * e * (2 if case["add"] else 1) + (4 * n if case["bias"] else 0),
                "flops": 2 * m * n * k + 3 * m * k}
    lens = _lengths(case)
    keys = sum(lens)
    rows = case["queries"] * case["heads"]
    return {"bytes": 2 * case["batch"] * rows * case["d"] * e + 4 * case["batch"] * rows + 2 * keys * case["key_heads"] * case["d"] * e
            + (keys if case["masked"] else 0),
            "flops": rows * keys * (4 * case["d"] + 4)}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _to_e4m3(y):
    """y (64 bits, at most 448 in magnitude) to the nearest number of a 4-bit exponent and a 3-bit mantissa, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _quantized64(x, tile):
    """(values in 8 bits, scale of each element's block, scales) in 64 bits."""
    x = x.double()
    size = torch.nn.functional.max_pool2d(x.abs()[None, None], (tile, BLOCK), ceil_mode=True)[0, 0]
    scale = torch.ones_like(size)
    some = size > 0
    scale[some] = torch.exp2(torch.ceil(torch.log2(size[some] / 448.0)))
    scale = torch.where(size > 448.0 * scale, 2 * scale, scale)              # (a logarithm next to a whole number may be off)
    scale = torch.where(some & (size <= 224.0 * scale), scale / 2, scale)
    each = scale.repeat_interleave(tile, 0)[: x.shape[0]].repeat_interleave(BLOCK, 1)[:, : x.shape[1]]
    return _to_e4m3(x / each), each, scale


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        parts = [_quantized64(s["x"][i: i + 32768], case["tile"]) for i in range(0, case["rows"], 32768)]
        return {"x8": torch.cat([y for y, _, _ in parts]), "scale": torch.cat([x for _, _, x in parts])}
    if case["op"] == "project":
        n, k = case["n"], case["k"]
        each = s["w_scale"].double().repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)[:, :k]
        w = s["w"].double() * each
        out = torch.empty(case["m"], n, device=DEV, dtype=torch.float64)
        for i in range(0, case["m"], 16384):
            y, scale, _ = _quantized64(s["x"][i: i + 16384], 1)
            out[i: i + 16384] = torch.nn.functional.linear(y * scale, w)
        if s["bias"] is not None:
            out += s["bias"].double()
        if s["add"] is not None:
            out += s["add"].double()
        return out
    b, lq, h, hk, d = case["batch"], case["queries"], case["heads"], case["key_heads"], case["d"]
    out = torch.zeros(b, lq, h, d, device=DEV, dtype=torch.float64)
    lse = torch.full((b, lq, h), -math.inf, device=DEV, dtype=torch.float64)
    start = 0
    for i, n in enumerate(_lengths(case)):
        pick = (lambda x: x[start: start + n]) if case["packed"] else (lambda x: x[i, :n])
        k, v = pick(s["k"]).double(), pick(s["v"]).double()
        if s["mask"] is not None:
            k, v = k[pick(s["mask"])], v[pick(s["mask"])]
        start += n
        if k.shape[0] == 0:
            continue
        for j in range(h):
            z = torch.einsum("qd,kd->qk", s["q"][i, :, j].double(), k[:, j // (h // hk)]) * s["scale"]
            lse[i, :, j] = torch.logsumexp(z, -1)
            out[i, :, j] = torch.exp(z - lse[i, :, j, None]) @ v[:, j // (h // hk)]
    return {"out": out, "lse": lse}
