"""What is measured of the token-wise operators: the gated delta rule over packed sequences (`token_scan`) and for a few
tokens a request (`token_step`), and rotary positions on time, height and width (`rotate`).

`run` computes them in elementary torch operations, or, where `own` is set, through the library's binding.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
CHUNK = 64


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the text state of one 768p-shaped layer: a single short prompt through all 40 heads
        dict(name="scan prompt 77", op="scan", dtype="bf16", d=128, heads=40, key_heads=40, tokens=77, seqs=1, split=0,
             start=False, l2=False),
        # prompts of uneven lengths packed one behind another, two value heads to a key head, going on from stored states
        dict(name="scan prompts 13", op="scan", dtype="bf16", d=128, heads=32, key_heads=16, tokens=5003, seqs=13, split=3,
             start=True, l2=True),
        # a full batch of documents: as many chains as keep the whole GPU busy
        dict(name="scan batch 32", op="scan", dtype="bf16", d=128, heads=32, key_heads=16, tokens=65536, seqs=32, split=5,
             start=False, l2=True),
        # the 480p-shaped clip token by token: one long sequence, few heads
        dict(name="scan clip 480p", op="scan", dtype="bf16", d=128, heads=8, key_heads=8, tokens=32760, seqs=1, split=0,
             start=True, l2=False),
        # the tiny configuration in 32 bits
        dict(name="scan f32 tiny", op="scan", dtype="f32", d=64, heads=2, key_heads=2, tokens=256, seqs=1, split=0,
             start=True, l2=False),
        # the scan-depth sweep's clip token by token: the longest sequence
        dict(name="scan sweep 262144", op="scan", dtype="bf16", d=128, heads=24, key_heads=24, tokens=262144, seqs=1,
             split=0, start=False, l2=False),
        # one user, one token: latency
        dict(name="step one", op="step", dtype="bf16", d=128, heads=40, key_heads=40, requests=1, per=1, slots=4, l2=True),
        # a serving batch, one token each, states anywhere in a larger pool
        dict(name="step batch 256", op="step", dtype="bf16", d=128, heads=32, key_heads=16, requests=256, per=1, slots=300,
             l2=True),
        # a few tokens a request (a draft being taken over), 32 bits, an odd batch
        dict(name="step f32 4 tokens", op="step", dtype="f32", d=64, heads=12, key_heads=4, requests=33, per=4, slots=40,
             l2=False),
        # the tiny configuration's queries and keys in 32 bits: latency
        dict(name="rotate tiny", op="rotate", dtype="f32", d=64, heads=2, key_heads=2, batch=1, frames=4, rows=8, cols=8,
             half=False, explicit=False, norm=False),
        # the 480p-shaped clip, split-halves pairs, positions given by the caller, heads normalised first, fewer key heads
        dict(name="rotate 480p", op="rotate", dtype="bf16", d=128, heads=8, key_heads=2, batch=1, frames=21, rows=30,
             cols=52, half=True, explicit=True, norm=True),
        # the 768p-shaped clip, neighbouring pairs, positions from the grid
        dict(name="rotate 768p", op="rotate", dtype="bf16", d=128, heads=40, key_heads=40, batch=1, frames=86, rows=48,
             cols=85, half=False, explicit=False, norm=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("scan", "scan", "step", "rotate"))
    f32 = rng.random() < 0.25
    d = 64 if rng.random() < 0.25 else 128
    key_heads = rng.choice((1, 2, 3, 4, 8, 12))
    heads = key_heads * rng.choice((1, 1, 2, 3))
    base = dict(op=op, dtype="f32" if f32 else "bf16", d=d, heads=heads, key_heads=key_heads)
    if op == "scan":
        fast = not f32 and d == 128
        tokens = _log_int(rng, 1, min(200000, 2500000 // heads) if fast else 9000)
        seqs = min(tokens, _log_int(rng, 1, 64))
        return dict(base, tokens=tokens, seqs=seqs, split=rng.randrange(1, 1000), start=rng.random() < 0.5,
                    l2=rng.random() < 0.5)
    if op == "step":
        requests = _log_int(rng, 1, 300)
        return dict(base, requests=requests, per=rng.choice((1, 1, 1, 2, 3, 5)), slots=requests + rng.randrange(0, 60),
                    l2=rng.random() < 0.5)
    return dict(base, batch=rng.choice((1, 1, 2)), frames=_log_int(rng, 1, 90), rows=_log_int(rng, 1, 48),
                cols=_log_int(rng, 1, 85), half=rng.random() < 0.5, explicit=rng.random() < 0.5, norm=rng.random() < 0.5)


def _lengths(case):
    """Token counts of a packed batch: uneven, some of them zero."""
    n, s = case["tokens"], case["seqs"]
    if s == 1:
        return [n]
    r = random.Random(case["split"])
    share = [r.random() ** 2 for _ in range(s)]
    total = sum(share) or 1.0
    cuts, acc = [0], 0.0
    for x in share[:-1]:
        acc += x
        cuts.append(min(n, int(n * acc / total)))
    cuts.append(n)
    return [b - a for a, b in zip(cuts, cuts[1:])]


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _tokens(gen, case, n):
    """q, k, v, beta, log_alpha of n tokens: keys partly near a few shared directions, the decay of each head at a time
    scale of its own (from a few tokens to thousands)."""
    d, h, hk, dt = case["d"], case["heads"], case["key_heads"], _dtype(case)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    q, k = rand(n, hk, d), rand(n, hk, d)
    shared = unit(rand(8, hk, d))
    near = torch.rand(n, hk, 1, generator=gen, device=DEV) < 0.3
    which = torch.randint(0, 8, (n,), generator=gen, device=DEV)
    k = torch.where(near, shared[which] * math.sqrt(d) + 0.4 * k, k)
    if not case["l2"]:
        q, k = unit(q), unit(k)
    v = rand(n, h, d)
    beta = torch.sigmoid(rand(n, h))
    rate = 1.0 + 15.0 * torch.rand(h, generator=gen, device=DEV)
    dt0 = torch.exp(torch.empty(h, device=DEV).uniform_(math.log(1e-3), math.log(0.1), generator=gen))
    bias = dt0 + torch.log(-torch.expm1(-dt0))
    log_alpha = -rate * torch.nn.functional.softplus(rand(n, h) + bias)
    return dict(q=q.to(dt), k=k.to(dt), v=v.to(dt), beta=beta, log_alpha=log_alpha)


def _pairs(case):
    """(angular frequency, axis) of each rotated pair: about a quarter of the pairs on time, the rest on height and width."""
    n = case["d"] // 2
    t = n // 4
    y = (n - t) // 2
    sections = (t, y, n - t - y)
    freq = [10000.0 ** (-i / c) for c in sections for i in range(c)]
    axis = [a for a, c in enumerate(sections) for _ in range(c)]
    return torch.tensor(freq, dtype=torch.float64), torch.tensor(axis, dtype=torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case=case, scale=case["d"] ** -0.5)
    h, d = case["heads"], case["d"]
    if case["op"] == "scan":
        s.update(_tokens(gen, case, case["tokens"]))
        lens = _lengths(case)
        s["max_len"] = max(lens)
        s["cu_seqlens"] = torch.tensor([0] + lens).cumsum(0).to(torch.int32).to(DEV)
        s["s0"] = 0.3 * torch.randn(case["seqs"], h, d, d, generator=gen, device=DEV) if case["start"] else None
    elif case["op"] == "step":
        x = _tokens(gen, case, case["requests"] * case["per"])
        s.update({n: t.view(case["requests"], case["per"], *t.shape[1:]) for n, t in x.items()})
        s["state"] = 0.3 * torch.randn(case["slots"], h, d, d, generator=gen, device=DEV)
        s["index"] = torch.randperm(case["slots"], generator=gen, device=DEV)[: case["requests"]].to(torch.int32)
    else:
        shape = (case["batch"], case["frames"], case["rows"] * case["cols"])
        dt, hk = _dtype(case), case["key_heads"]
        s["q"] = torch.randn(*shape, h, d, generator=gen, device=DEV, dtype=dt)
        s["k"] = torch.randn(*shape, hk, d, generator=gen, device=DEV, dtype=dt)
        s["freq"], s["axis"] = (x.to(DEV) for x in _pairs(case))
        s["positions"] = None
        if case["explicit"]:  # video tokens behind a text of its own length, in a long stream
            n = shape[0] * shape[1] * shape[2]
            s["positions"] = torch.randint(0, 100000, (3, n), generator=gen, device=DEV, dtype=torch.int32)
        s["wq"] = s["wk"] = None
        if case["norm"]:
            s["wq"] = 1 + 0.1 * torch.randn(d, generator=gen, device=DEV)
            s["wk"] = 1 + 0.1 * torch.randn(d, generator=gen, device=DEV)
    if own:
        from paper_2609_20744_b200 import binding
        s["vda"] = binding.Vda(d, case["dtype"])
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    op = s["case"]["op"]
    if own:
        return _own(s, op)
    return {"scan": _scan, "step": _step, "rotate": _rotate}[op](s)


def _own(s, op):
    eps = 1e-6 if s["case"].get("l2") else 0.0
    if op == "scan":
        out, state = s["vda"].token_scan(s["q"], s["k"], s["v"], s["beta"], log_alpha=s["log_alpha"],
                                         cu_seqlens=s["cu_seqlens"], s0=s["s0"], scale=s["scale"], l2_eps=eps)
        return {"out": out, "state": state}
    if op == "step":
        out = s["vda"].token_step(s["q"], s["k"], s["v"], s["beta"], s["state"], log_alpha=s["log_alpha"],
                                  index=s["index"], scale=s["scale"], l2_eps=eps)
        return {"out": out, "state": s["state"]}
    c = s["case"]
    q, k = s["vda"].rotate(s["q"], s["k"], s["freq"], s["axis"], c["rows"], c["cols"], positions=s["positions"],
                           half=c["half"], q_weight=s["wq"], k_weight=s["wk"], norm_eps=1e-6 if c["norm"] else 0.0)
    return {"q": q, "k": k}


# ------------------------------------------------------------------------------------------------ plain forms
def _features(s, axis):
    """q, k, v in 32 bits, normalised if the case asks for it, key heads repeated for their value heads."""
    c = s["case"]
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    if c["l2"]:
        q = q * torch.rsqrt(q.square().sum(-1, keepdim=True) + 1e-6)
        k = k * torch.rsqrt(k.square().sum(-1, keepdim=True) + 1e-6)
    r = c["heads"] // c["key_heads"]
    return q.repeat_interleave(r, axis), k.repeat_interleave(r, axis), v


def _unit_lower_inverse(lower):
    """(I + lower)^-1 of strictly lower 64 x 64 matrices, blocks of 1, 2, 4, ... merged pairwise."""
    n = lower.shape[0]
    inv = torch.eye(CHUNK, device=lower.device, dtype=lower.dtype).repeat(n, 1, 1)
    b = 1
    while b < CHUNK:
        m = CHUNK // (2 * b)
        i = torch.arange(m, device=lower.device)
        iv, lv = inv.view(n, m, 2 * b, m, 2 * b), lower.view(n, m, 2 * b, m, 2 * b)
        first, second = iv[:, i, :b, i, :b], iv[:, i, b:, i, b:]
        iv[:, i, b:, i, :b] = -(second @ lv[:, i, b:, i, :b] @ first)
        b *= 2
    return inv


def _scan(s):
    c = s["case"]
    h, d, seqs = c["heads"], c["d"], c["seqs"]
    chunks = max(1, -(-s["max_len"] // CHUNK))
    n = chunks * CHUNK
    start = s["cu_seqlens"][:-1].long()
    length = s["cu_seqlens"][1:].long() - start
    at = torch.arange(n, device=DEV)
    there = at[None] < length[:, None]                                     # [seqs, n]
    row = (start[:, None] + at[None]).clamp(max=c["tokens"] - 1)

    def padded(x):                                                         # [N, h, ...] -> [chunks, seqs*h, 64, ...]
        x = torch.where(there.view(seqs, n, *([1] * (x.dim() - 1))), x[row], torch.zeros((), device=DEV, dtype=x.dtype))
        x = x.view(seqs, chunks, CHUNK, h, *x.shape[3:])
        return x.movedim(3, 1).movedim(2, 0).reshape(chunks, seqs * h, CHUNK, *x.shape[4:])

    q, k, v = (padded(x) for x in _features(s, 1))
    beta, g = padded(s["beta"])[..., None], padded(s["log_alpha"]).double().cumsum(-1)
    low = torch.ones(CHUNK, CHUNK, device=DEV, dtype=torch.bool).tril()
    decay = torch.exp(torch.where(low, g[..., :, None] - g[..., None, :], 0.0)).float() * low
    lower = (beta * decay * (k @ k.mT)).tril(-1)
    inv = _unit_lower_inverse(lower.view(-1, CHUNK, CHUNK)).view_as(lower)
    mix = decay * (q @ k.mT)
    eg, last = torch.exp(g).float()[..., None], torch.exp(g[..., -1:] - g).float()[..., None]
    whole = torch.exp(g[..., -1]).float()[..., None, None]
    state = s["s0"].reshape(seqs * h, d, d).clone() if s["s0"] is not None else torch.zeros(seqs * h, d, d, device=DEV)
    out = torch.empty_like(v)
    for i in range(chunks):
        u = inv[i] @ (beta[i] * (v[i] - eg[i] * (k[i] @ state.mT)))
        out[i] = eg[i] * (q[i] @ state.mT) + mix[i] @ u
        state = whole[i] * state + (last[i] * u).mT @ k[i]
    out = out.view(chunks, seqs, h, CHUNK, d).permute(1, 0, 3, 2, 4).reshape(seqs, n, h, d)
    return {"out": (out[there] * s["scale"]).to(_dtype(c)), "state": state.view(seqs, h, d, d)}


def _step(s):
    q, k, v = _features(s, 2)
    index = s["index"].long()
    state = s["state"][index]
    out = torch.empty_like(v)
    for i in range(s["case"]["per"]):
        state = state * torch.exp(s["log_alpha"][:, i])[..., None, None]
        u = s["beta"][:, i, :, None] * (v[:, i] - (state @ k[:, i, :, :, None])[..., 0])
        state = state + u[..., :, None] * k[:, i, :, None, :]
        out[:, i] = (state @ q[:, i, :, :, None])[..., 0]
    s["state"][index] = state
    return {"out": (out * s["scale"]).to(_dtype(s["case"])), "state": s["state"]}


def _grid_positions(c):
    n = c["batch"] * c["frames"] * c["rows"] * c["cols"]
    at = torch.arange(n, device=DEV)
    u = at % (c["rows"] * c["cols"])
    return torch.stack(((at // (c["rows"] * c["cols"])) % c["frames"], u // c["cols"], u % c["cols"]))


def _rotate(s):
    c = s["case"]
    pos = s["positions"] if s["positions"] is not None else _grid_positions(c)
    angle = pos[s["axis"].long()].double() * s["freq"][:, None]            # [pairs, tokens]
    cos, sin = (f(angle).float().mT.reshape(*s["q"].shape[:3], 1, -1) for f in (torch.cos, torch.sin))

    def one(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
        n = cos.shape[-1]
        a, b = (x[..., :n], x[..., n:]) if c["half"] else (x[..., 0::2], x[..., 1::2])
        y, z = a * cos - b * sin, a * sin + b * cos
        r = torch.cat((y, z), -1) if c["half"] else torch.stack((y, z), -1).flatten(-2)
        return r.to(_dtype(c))

    return {"q": one(s["q"], s["wq"]), "k": one(s["k"], s["wk"])}


# ------------------------------------------------------------------------------------------------ floors
def work(case):
    d, h, hk = case["d"], case["heads"], case["key_heads"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "rotate":
        n = case["batch"] * case["frames"] * case["rows"] * case["cols"]
        return {"bytes": 2 * n * (h + hk) * d * e + (12 * n if case["explicit"] else 0),
                "flops": n * (h + hk) * d * (3 + (4 if case["norm"] else 0))}
    n = case["tokens"] if case["op"] == "scan" else case["requests"] * case["per"]
    tokens = n * (2 * hk * d * e + 2 * h * d * e + 8 * h)
    seqs = case["seqs"] if case["op"] == "scan" else case["requests"]
    states = seqs * h * d * d * 4 * (2 if case["op"] == "step" or case["start"] else 1)
    return {"bytes": tokens + states, "flops": n * h * 8 * d * d}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _rule64(q, k, v, beta, log_alpha, state, l2, scale):
    """The definition token by token: q, k [n, x, d], v [n, x, d], beta, log_alpha [n, x], state [x, d, d] (updated)."""
    if l2:
        q = q / torch.sqrt((q * q).sum(-1, keepdim=True) + 1e-6)
        k = k / torch.sqrt((k * k).sum(-1, keepdim=True) + 1e-6)
    out = torch.empty_like(v)
    alpha = torch.exp(log_alpha)[..., None, None]
    for kt, qt, vt, bt, at, ot in zip(k[..., None], q[..., None], v[..., None], beta[..., None, None], alpha, out):
        state.mul_(at)
        u = bt * (vt - torch.bmm(state, kt))
        state.baddbmm_(u, kt.mT)
        ot.copy_(torch.bmm(state, qt)[..., 0])
    return out * scale


def exact(case, seed):
    if case["op"] == "scan" and max(_lengths(case)) > 300000:
        return None
    s = prepare(case, seed)
    h, d = case["heads"], case["d"]
    if case["op"] == "rotate":
        return _rotate64(s, case)
    r = h // case["key_heads"]
    q, k, v, beta, g = (s[n].double() for n in ("q", "k", "v", "beta", "log_alpha"))
    q, k = q.repeat_interleave(r, -2), k.repeat_interleave(r, -2)
    if case["op"] == "step":
        at = s["index"].long()
        state = s["state"].double()
        some = state[at].flatten(0, 1)
        out = _rule64(*(x.movedim(1, 0).flatten(1, 2) for x in (q, k, v, beta, g)), some, case["l2"], s["scale"])
        state[at] = some.view(-1, h, d, d)
        return {"out": out.view(case["per"], case["requests"], h, d).movedim(0, 1), "state": state}
    state = torch.zeros(case["seqs"], h, d, d, device=DEV, dtype=torch.float64)
    if s["s0"] is not None:
        state += s["s0"]
    out = torch.zeros(case["tokens"], h, d, device=DEV, dtype=torch.float64)
    lens = _lengths(case)
    order = sorted(range(len(lens)), key=lambda i: -lens[i])              # the longest first: fewer go on at each token
    first = [sum(lens[:i]) for i in range(len(lens))]
    state = state[torch.tensor(order, device=DEV)]
    done = 0
    for stop in sorted(set(lens)):                                        # all sequences that are at least `stop` long
        live = [i for i in order if lens[i] >= stop]
        if stop > done and live:
            rows = torch.tensor([first[i] for i in live], device=DEV)[None] + torch.arange(done, stop, device=DEV)[:, None]
            part = state[: len(live)].flatten(0, 1)
            o = _rule64(*(x[rows].flatten(1, 2) for x in (q, k, v, beta, g)), part, case["l2"], s["scale"])
            out[rows] = o.view(stop - done, len(live), h, d)
            state[: len(live)] = part.view(len(live), h, d, d)
        done = stop
    back = torch.empty_like(state)
    back[torch.tensor(order, device=DEV)] = state
    return {"out": out, "state": back}


def _rotate64(s, case):
    """Each pair as a complex number times e^{i angle}, frame by frame."""
    rows, cols, frames = case["rows"], case["cols"], case["frames"]
    given = s["positions"].view(3, case["batch"], frames, -1) if s["positions"] is not None else None
    u = torch.arange(rows * cols, device=DEV)
    result = {}
    for name, w in (("q", s["wq"]), ("k", s["wk"])):
        y = torch.empty(s[name].shape, device=DEV, dtype=torch.float64)
        for b in range(case["batch"]):
            for t in range(frames):
                p = given[:, b, t] if given is not None else torch.stack((torch.full_like(u, t), u // cols, u % cols))
                turn = torch.polar(torch.ones((), device=DEV, dtype=torch.float64),
                                   torch.stack([p[a].double() * f for a, f in zip(s["axis"].tolist(), s["freq"])], -1))[:, None]
                x = s[name][b, t].double()
                if w is not None:
                    x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.double()
                if case["half"]:
                    z = torch.complex(*x.chunk(2, -1)) * turn
                    y[b, t] = torch.cat((z.real, z.imag), -1)
                else:
                    y[b, t] = torch.view_as_real(torch.view_as_complex(x.unflatten(-1, (-1, 2)).contiguous()) * turn).flatten(-2)
        result[name] = y
    return result
