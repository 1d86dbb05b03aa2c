"""token_scan, token_step and rotate against their 64-bit statements.

Tolerances, all relative in the 2-norm over one (sequence or request, head) slice.  u16 = 2^-8 (half a step of bf16), u32 = 2^-24.
  state, plain-fp32 kernels: a token's two d-long dot products in eight partial sums of d/8 terms, three shuffle steps and
     about eight further operations round (d/8 + 11) times u32 at most, relative to the state; the roundings of n
     tokens are independent:  (d/8 + 11) sqrt(n) u32.
  state, tensor cores: the state, the differences X, the operator E and the triangular inverse are each cut to two bf16
     parts, off by at most u16^2 = 2^-16 of the value:  4 * 2^-16, plus the fp32 term above.
  out: one rounding to io_dtype, u16 (u32 for fp32) of the value.  Further errors -- the state's, and on the tensor cores
     those of the state, X and the mixing matrix, allowed 3 u16 here -- are roundings of the terms S_ij q_j, which may
     cancel in their sum: independent, they are relative to the root of the terms' summed squares (the oracle's `sizes`),
     not to the result.  (A rank-one state read by a query at right angles to its key gives next to nothing.)  The tensor
     cores' two parts of each factor give far less than 3 u16: test_scan_readout_with_keys_alike.
"""
import numpy as np
import pytest
import torch

from oracle import token_oracle as tok
from oracle import vda_oracle as orc
from paper_2609_20744_b200 import binding, build, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U16, U32 = 2.0 ** -8, 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.load_library()


def np64(x):
    return None if x is None else x.detach().double().cpu().numpy()


def draw(n, h, hk, d, dtype, seed=0, l2=False, near=0.3, decay=True):
    """Tokens as a layer meets them: unit keys, some near a few shared directions, a decay per head from fast to none."""
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    shared = unit(rand(4, hk, d))
    k = unit(torch.where(torch.rand(n, hk, 1, generator=g) < near, shared[torch.randint(0, 4, (n,), generator=g)] + 0.05 * rand(n, hk, d),
                         unit(rand(n, hk, d))))
    q = unit(rand(n, hk, d))
    if l2:
        q, k = 3 * q, 0.5 * k
    x = dict(q=q, k=k, v=rand(n, h, d), beta=torch.sigmoid(rand(n, h)))
    x["log_alpha"] = -torch.exp(rand(n, h) - 3 - torch.arange(h)) if decay else None
    for name in ("q", "k", "v"):
        x[name] = x[name].to(TYPES[dtype])
    return {n: t.to(DEV) if t is not None else None for n, t in x.items()}


def tensor_cores(dtype, d, flags=0):
    return dtype == "bf16" and d == 128 and not flags & binding.VDN_FLAG_FORCE_SIMT


def tolerances(dtype, d, n, tc):
    state = (d / 8 + 11) * max(1, n) ** 0.5 * U32 + (4 * 2.0 ** -16 if tc else 0)
    return U32 if dtype == "f32" else U16, state + (3 * U16 if tc else 0), state


def out_ok(got, want, sizes, tol):
    """got, want [n, d] of one head, sizes [n]; tol from tolerances()."""
    return np.linalg.norm(np64(got) - want) <= tol[0] * np.linalg.norm(want) + tol[1] * np.linalg.norm(sizes)


def rel(got, want):
    got, want = np64(got) if torch.is_tensor(got) else got, np.asarray(want)
    off = np.linalg.norm(got - want)
    return off / np.linalg.norm(want) if np.linalg.norm(want) else off


def check_scan(vda, x, lens, dtype, d, tc, s0=None, scale=1.0, l2_eps=0.0, out=None, state=None, walks=1, **kw):
    cu = torch.tensor([0] + list(lens)).cumsum(0).to(torch.int32).to(DEV)
    sizes = []
    want_o, want_s = tok.packed(np64(x["q"]), np64(x["k"]), np64(x["v"]), np64(x["beta"]), lens, np64(x["log_alpha"]),
                                np64(s0), scale, l2_eps, sizes)
    sizes = np.array(sizes).reshape(sum(lens), x["v"].shape[1])
    out, state = vda.token_scan(**x, cu_seqlens=cu, s0=s0, scale=scale, l2_eps=l2_eps, out=out, state=state, **kw)
    torch.cuda.synchronize()
    assert vda.status() == binding.VDN_OK
    at = 0
    for i, n in enumerate(lens):
        tol = tolerances(dtype, d, walks * n, tc)
        w = slice(at, at + n)
        for h in range(state.shape[1]):
            assert rel(state[i, h], want_s[i, h]) <= tol[2], (i, h, n)
            assert out_ok(out[w, h], want_o[w, h], sizes[w, h], tol), (i, h, n)
        at += n
    return out, state


# (the last three, and [128] and [300], are long enough on the whole that bf16 with d = 128 goes in chunks)
LENS = [[1], [2], [63], [64], [65], [128], [300], [5, 0, 64, 1, 130, 0, 63], [0], [1, 400, 0, 64, 65, 63, 2], [129, 0, 1, 191], [700]]


@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("dtype,d,flags", [("f32", 64, 0), ("f32", 128, 0), ("bf16", 64, 0), ("bf16", 128, 0),
                                           ("bf16", 128, binding.VDN_FLAG_FORCE_SIMT)])
def test_scan(dtype, d, flags, lens):
    h, hk = (4, 2) if sum(lens) % 2 else (3, 3)
    vda = binding.Vda(d, dtype, flags=flags)
    x = draw(sum(lens), h, hk, d, dtype, seed=len(lens))
    s0 = 0.3 * torch.randn(len(lens), h, d, d, device=DEV) if len(lens) > 1 or lens[0] % 3 == 0 else None
    check_scan(vda, x, lens, dtype, d, tensor_cores(dtype, d, flags), s0, scale=0.5)


@pytest.mark.parametrize("length", [1.0, 1.3])
@pytest.mark.parametrize("keys", ["same", "two", "near"])
def test_scan_readout_with_keys_alike(keys, length):
    """Chunks whose operators cancel: keys alike, beta = 1.  Per chunk of 64, O = e^G S q + P X with P = M T, M the decayed q.k, T the
    inverse of I + L.  Every factor but q and k has two bf16 parts, off by u16^2 = 2^-16, and the accumulators are fp32: the
    result is off by u16 of itself, by 2^-16 of each of S, X, M, T and P's terms, taken without their signs, and by what the state
    is off, at most the state's tolerance of its norm (and of X's, which has it as e^G S k)."""
    d, h, n, C = 128, 2, 320, 64
    x = draw(n, h, h, d, "bf16", seed=15)
    unit = lambda t: t / t.norm(dim=-1, keepdim=True)  # noqa: E731
    g = torch.Generator().manual_seed(16)
    shared = unit(torch.randn(4, h, d, generator=g))
    pick = torch.randint(0, {"same": 1, "two": 2, "near": 4}[keys], (n,), generator=g)
    k = shared[pick] if keys != "near" else unit(shared[pick] + 0.05 * unit(torch.randn(n, h, d, generator=g)))
    x["k"] = (length * k).to(torch.bfloat16).to(DEV)
    x["beta"] = torch.ones(n, h, device=DEV)
    x["log_alpha"] = -1e-3 * torch.rand(n, h, generator=g).to(DEV)
    got, state = binding.Vda(d, "bf16").token_scan(**x)
    q, k, v, beta, ga = (x[name].double().cpu() for name in ("q", "k", "v", "beta", "log_alpha"))
    for j in range(h):
        S, want, off = torch.zeros(d, d, dtype=torch.float64), [], []
        for c in range(0, n, C):
            Q, K, V, b, G = q[c:c + C, j], k[c:c + C, j], v[c:c + C, j], beta[c:c + C, j], ga[c:c + C, j].cumsum(0)
            decay = torch.exp(G[:, None] - G[None]).tril()
            T = torch.linalg.inv(torch.eye(C, dtype=torch.float64) + (b[:, None] * decay * (K @ K.T)).tril(-1)) * b[None]
            M, X, e = decay * (Q @ K.T), V - torch.exp(G)[:, None] * (K @ S.T), torch.exp(G)[:, None]
            want.append(e * (Q @ S.T) + M @ T @ X)
            P = M.abs() @ T.abs()                     # what the parts of M and of T are relative to
            eps, tol = 2.0 ** -16, 4 * 2.0 ** -16 * length ** 2
            from_state = tol * float(S.norm()) * (e * Q.norm(dim=1, keepdim=True) + (P @ (e * K.norm(dim=1, keepdim=True))))
            off.append(eps * (e * (Q.abs() @ S.abs().T) + 4 * (P @ X.abs())) + from_state / d ** 0.5)
            S = torch.exp(G[-1]) * S + (T @ X).T @ (torch.exp(G[-1] - G)[:, None] * K)
        want, off = torch.cat(want), torch.cat(off)
        assert float((got[:, j].double().cpu() - want).norm()) <= U16 * float(want.norm()) + float(off.norm())


@pytest.mark.parametrize("dtype,d,flags", [("f32", 64, 0), ("f32", 128, 0), ("bf16", 64, 0),
                                           ("bf16", 128, binding.VDN_FLAG_FORCE_SIMT)])
def test_scan_of_more_rows_than_run_at_once(dtype, d, flags):
    """The plain kernel gives a CTA more rows where there are many sequences and heads."""
    lens = [9, 17, 34, 0, 1, 63] * 5
    x = draw(sum(lens), 4, 2, d, dtype, seed=11)
    s0 = 0.3 * torch.randn(len(lens), 4, d, d, device=DEV)
    check_scan(binding.Vda(d, dtype, flags=flags), x, lens, dtype, d, False, s0, scale=0.5)


@pytest.mark.parametrize("dtype,d,flags", [("f32", 64, 0), ("f32", 128, 0), ("bf16", 64, 0),
                                           ("bf16", 128, binding.VDN_FLAG_FORCE_SIMT)])
@pytest.mark.parametrize("lens", [[1000], [131, 0, 1203, 64], [577, 578]], ids=str)
def test_scan_plain_in_parts(dtype, d, flags, lens):
    """Few long sequences, cut into parts.  Three walks (what a part writes, what it makes of an entering state, the part itself) each
    add a rounding a token, the joins one product of d terms a part of 64 tokens or more: fewer than four walks' roundings."""
    vda = binding.Vda(d, dtype, flags=flags)
    x = draw(sum(lens), 2, 1, d, dtype, seed=12)
    x["log_alpha"][200] = -float("inf")
    s0 = 0.3 * torch.randn(len(lens), 2, d, d, device=DEV)
    vda.profile(True)
    check_scan(vda, x, lens, dtype, d, False, s0, scale=0.5, state=s0, walks=4)
    assert [k[0] for k in vda.kernel_times()] == ["token_coef", "token_walk_compose", "token_join", "token_walk"]


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 64), ("bf16", 128)])
def test_scan_normalises_queries_and_keys(dtype, d):
    x = draw(200, 4, 2, d, dtype, seed=3, l2=True)
    check_scan(binding.Vda(d, dtype), x, [70, 130], dtype, d, tensor_cores(dtype, d), l2_eps=1e-6, scale=d ** -0.5)


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
@pytest.mark.parametrize("case", ["no decay", "forget", "strong decay", "beta 0", "beta 1", "same key"])
def test_scan_gates(dtype, d, case):
    n, h = 190, 3
    x = draw(n, h, h, d, dtype, seed=4, decay=case != "no decay")
    if case == "forget":                     # document borders inside a sequence, one in the middle of a chunk, two in a row
        x["log_alpha"][[0, 20, 64, 100, 101]] = -float("inf")
    elif case == "strong decay":
        x["log_alpha"] = -50 * torch.rand(n, h, device=DEV)
    elif case == "beta 0":
        x["beta"][:] = 0
    elif case == "beta 1":
        x["beta"][:] = 1
    elif case == "same key":
        x["k"][:] = x["k"][:1].clone()
    s0 = torch.randn(1, h, d, d, device=DEV)
    check_scan(binding.Vda(d, dtype), x, [n], dtype, d, tensor_cores(dtype, d), s0)


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
def test_scan_leaves_rows_behind_the_last_sequence_and_does_not_read_them(dtype, d):
    lens, extra, h = [33, 64, 20], 50, 2
    n = sum(lens) + extra
    x = draw(n, h, h, d, dtype, seed=5)
    for t in ("q", "k", "v", "beta", "log_alpha"):
        x[t][n - extra:] = float("nan")
    x["v"][n - extra + 1] = float("inf")
    out = torch.full((n, h, d), 7.0, device=DEV, dtype=TYPES[dtype])
    check_scan(binding.Vda(d, dtype), x, lens, dtype, d, tensor_cores(dtype, d), out=out)
    assert (out[n - extra:] == 7).all()


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
def test_scan_values_of_one_sequence_do_not_reach_its_neighbours(dtype, d):
    """A sequence full of NaN between two others, ending inside a chunk."""
    lens, h = [70, 30, 70], 2
    x = draw(sum(lens), h, h, d, dtype, seed=6)
    cu = torch.tensor([0, 70, 100, 170], dtype=torch.int32, device=DEV)
    vda = binding.Vda(d, dtype)
    clean_o, clean_s = vda.token_scan(**x, cu_seqlens=cu)
    for t in ("q", "k", "v", "beta", "log_alpha"):
        x[t][70:100] = float("nan")
    out, state = vda.token_scan(**x, cu_seqlens=cu)
    keep = torch.cat([torch.arange(70), torch.arange(100, 170)]).to(DEV)
    assert torch.equal(out[keep], clean_o[keep]) and torch.equal(state[[0, 2]], clean_s[[0, 2]])
    assert out[70:100].isnan().all() and state[1].isnan().all()


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
def test_scan_of_slices_in_place_states_and_another_stream(dtype, d):
    h, hk, lens = 4, 2, [100, 61]
    n = sum(lens)
    x = draw(n, h, hk, d, dtype, seed=7)
    both = torch.cat([x["q"], x["k"], x["v"]], 1)
    x["q"], x["k"], x["v"] = both[:, :hk], both[:, hk:2 * hk], both[:, 2 * hk:]
    wide = torch.full((n, 2 * h, d), 3.0, device=DEV, dtype=TYPES[dtype])
    s0 = torch.randn(2, h, d, d, device=DEV)
    vda = binding.Vda(d, dtype)
    want_o, want_s = vda.token_scan(**x, cu_seqlens=torch.tensor([0, 100, n], dtype=torch.int32, device=DEV), s0=s0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out, state = check_scan(vda, x, lens, dtype, d, tensor_cores(dtype, d), s0.clone(), out=wide[:, h:], stream=side)
    assert torch.equal(out, want_o) and torch.equal(state, want_s) and (wide[:, :h] == 3).all()
    state = s0.clone()
    vda.token_scan(**x, cu_seqlens=torch.tensor([0, 100, n], dtype=torch.int32, device=DEV), s0=state, state=state)
    assert torch.equal(state, want_s)


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
def test_scan_captured_twice_and_replayed_on_new_inputs(dtype, d):
    """Two graphs of one handle, replayed in turn on two streams, each with a workspace of its own."""
    h = 2
    vda = binding.Vda(d, dtype)
    runs = []
    for seed, lens in ((1, [90, 40]), (2, [17, 200])):
        x = draw(sum(lens), h, h, d, dtype, seed=seed)
        cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32).to(DEV)
        s0 = torch.randn(2, h, d, d, device=DEV)
        vda.token_scan(**x, cu_seqlens=cu, s0=s0)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = vda.token_scan(**x, cu_seqlens=cu, s0=s0)
        runs.append((g, x, cu, s0, got, draw(sum(lens), h, h, d, dtype, seed=seed + 10)))
    for _ in range(2):
        for g, x, cu, s0, got, new in runs:
            for name in x:
                x[name].copy_(new[name])
            s0.mul_(0.5)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in runs]
        for r, st in zip(runs, streams):
            with torch.cuda.stream(st):
                r[0].replay()
        torch.cuda.synchronize()
        for g, x, cu, s0, got, new in runs:
            o, s = vda.token_scan(**x, cu_seqlens=cu, s0=s0)
            assert torch.equal(o, got[0]) and torch.equal(s, got[1])


@pytest.mark.parametrize("tokens,h", [(6000, 2), (20011, 1)])
def test_scan_long_sequence_on_the_tensor_cores_agrees_with_the_plain_kernel(tokens, h):
    """Long enough that a sequence is cut into parts that run side by side; a short one beside it is not."""
    d = 128
    x = draw(tokens, h, h, d, "bf16", seed=8)
    cu = torch.tensor([0, tokens - 100, tokens], dtype=torch.int32, device=DEV)
    s0 = torch.randn(2, h, d, d, device=DEV)
    o1, s1 = binding.Vda(d, "bf16").token_scan(**x, cu_seqlens=cu, s0=s0)
    o2, s2 = binding.Vda(d, "bf16", flags=binding.VDN_FLAG_FORCE_SIMT).token_scan(**x, cu_seqlens=cu, s0=s0)
    # both off by their own bounds; a read-out of many tokens' state is as large as its terms
    io, terms, state = tolerances("bf16", d, tokens, True)
    assert rel(s1, np64(s2)) <= 2 * state and rel(o1, np64(o2)) <= 2 * (io + terms)


@pytest.mark.parametrize("lens,h,hk", [([1000], 5, 5), ([700, 1300, 64, 1, 900] * 6, 32, 16), ([9000], 8, 8)], ids=str)
def test_scan_same_call_same_bits(lens, h, hk):
    """Over and over, calls right behind one another, on every SM: what a missing wait between two roles of a kernel would break."""
    d, n = 128, sum(lens)
    x = draw(n, h, hk, d, "bf16", seed=9)
    cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32).to(DEV)
    vda = binding.Vda(d, "bf16")
    o1, s1 = vda.token_scan(**x, cu_seqlens=cu)
    for _ in range(5):
        many = [vda.token_scan(**x, cu_seqlens=cu) for _ in range(4)]
        assert all(torch.equal(o, o1) and torch.equal(s, s1) for o, s in many)
    io, terms, state = tolerances("bf16", d, max(lens), True)
    o2, s2 = binding.Vda(d, "bf16", flags=binding.VDN_FLAG_FORCE_SIMT).token_scan(**x, cu_seqlens=cu)
    # token by token of each head: the largest difference of a row counts, not the mean over all
    off = (o1.double() - o2.double()).norm(dim=-1) / o2.double().norm(dim=(0, 2))[None] * n ** 0.5
    assert float(off.max()) <= 8 * (io + terms)          # rows are up to a few times the mean row
    assert rel(s1, np64(s2)) <= 2 * state


@pytest.mark.parametrize("dtype,d,lens,h", [("f32", 64, [2500], 2), ("f32", 128, [700, 3, 1300], 4), ("bf16", 64, [80] * 40, 8)],
                         ids=str)
def test_plain_scan_same_call_same_bits(dtype, d, lens, h):
    """The plain kernels likewise, in parts and whole, two calls of one handle at once on streams of their own among them."""
    x = draw(sum(lens), h, h, d, dtype, seed=13)
    cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32).to(DEV)
    vda = binding.Vda(d, dtype)
    o1, s1 = vda.token_scan(**x, cu_seqlens=cu)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        many = [vda.token_scan(**x, cu_seqlens=cu, stream=streams[i % 2]) for i in range(6)]
        torch.cuda.synchronize()
        assert all(torch.equal(o, o1) and torch.equal(s, s1) for o, s in many)


def test_scan_takes_the_kernels_its_sizes_call_for():
    """Short sequences token by token, longer ones in chunks, few long ones in parts."""
    d, h = 128, 2
    few, walk, chunks = ["token_few"], ["token_coef", "token_walk"], ["token_prep", "token_chain"]
    parts = ["token_prep", "token_compose", "token_join", "token_chain"]
    plain_parts = ["token_coef", "token_walk_compose", "token_join", "token_walk"]
    for flags, wanted in ((0, {2: few, 20: walk, 300: chunks, 3000: parts}),
                          (binding.VDN_FLAG_FORCE_SIMT, {2: few, 20: walk, 300: walk, 3000: plain_parts})):
        for n, names in wanted.items():
            vda = binding.Vda(d, "bf16", flags=flags)
            vda.profile(True)
            vda.token_scan(**draw(n, h, h, d, "bf16"))
            assert [k[0] for k in vda.kernel_times()] == names and vda.launch_count() == len(names)


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
def test_offsets_beyond_32_bits(dtype, d):
    """Slices of one wide buffer whose last rows lie more than 2^31 elements in, a pool of states likewise: the bits of dense tensors."""
    h, n, width = 2, 2150, 1 << 20
    if torch.cuda.mem_get_info(DEV)[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    x = draw(n, h, h, d, dtype, seed=14)
    vda = binding.Vda(d, dtype)
    wide = torch.empty(n, width, dtype=TYPES[dtype], device=DEV)
    part = {}
    for i, name in enumerate(("q", "k", "v", "out")):
        part[name] = wide[:, i * 1024:i * 1024 + h * d].view(n, h, d)
        if name != "out":
            part[name].copy_(x[name])
    assert (n - 1) * width > 2 ** 31
    o1, s1 = vda.token_scan(**x)
    o2, s2 = vda.token_scan(**{**x, **part})
    assert torch.equal(o2, o1) and torch.equal(s2, s1) and o2.data_ptr() == part["out"].data_ptr()
    # its last four rows as four requests
    slots = 2 ** 31 // (h * d * d) + 3
    pool = torch.empty(slots, h, d, d, device=DEV)
    index = torch.tensor([slots - 1, 0, slots - 2, 7], dtype=torch.int32, device=DEV)
    pool[index.long()] = s1
    few = {name: t[-4:] for name, t in x.items()}
    small = s1.expand(4, -1, -1, -1).contiguous()
    o1 = vda.token_step(**few, state=small)
    vda.token_step(**few, **{name: t[-4:] for name, t in part.items() if name == "out"}, state=pool, index=index)
    assert torch.equal(part["out"][-4:], o1) and torch.equal(pool[index.long()], small)
    del pool
    # one frame of all tokens, in place
    freq, axis = binding.rotary_tables((8, 8, 8))
    at = dict(freq=freq.to(DEV), axis=axis.to(DEV), Y=1, X=n)
    q1, k1 = vda.rotate(x["q"][None, None], x["k"][None, None], **at)
    q2, k2 = vda.rotate(part["q"][None, None], part["k"][None, None], out=(part["q"][None, None], part["k"][None, None]), **at)
    assert torch.equal(q2, q1) and torch.equal(k2, k1)


def test_scan_of_no_tokens():
    for dtype, d in (("f32", 64), ("bf16", 128)):
        x = draw(0, 2, 2, d, dtype)
        s0 = torch.randn(3, 2, d, d, device=DEV)
        out, state = binding.Vda(d, dtype).token_scan(**x, cu_seqlens=torch.zeros(4, dtype=torch.int32, device=DEV), s0=s0)
        assert out.shape == (0, 2, d) and torch.equal(state, s0)


# ---------------------------------------------------------------------------------------------------------------- step
@pytest.mark.parametrize("dtype,d", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("requests,per,h,hk", [(1, 1, 2, 2), (7, 1, 6, 2), (5, 3, 4, 4), (2, 40, 2, 1), (61, 2, 12, 4)])
def test_step(dtype, d, requests, per, h, hk):
    slots = requests + 3
    x = draw(requests * per, h, hk, d, dtype, seed=requests, l2=True)
    pool = 0.3 * torch.randn(slots, h, d, d, device=DEV)
    index = torch.randperm(slots)[:requests].to(torch.int32)
    before = pool.clone()
    shaped = {n: t.view(requests, per, *t.shape[1:]) if per > 1 else t for n, t in x.items()}
    vda = binding.Vda(d, dtype)
    out = vda.token_step(**shaped, state=pool, index=index.to(DEV), scale=0.7, l2_eps=1e-6).view(requests, per, h, d)
    torch.cuda.synchronize()
    assert vda.status() == binding.VDN_OK
    tol = tolerances(dtype, d, per, False)
    x = {n: np64(t) for n, t in x.items()}
    for r in range(requests):
        w, sizes = slice(r * per, (r + 1) * per), []
        o, s = tok.delta_rule(x["q"][w], x["k"][w], x["v"][w], x["beta"][w], x["log_alpha"][w], np64(before[index[r]]), 0.7, 1e-6, sizes)
        for i in range(h):
            assert rel(pool[index[r], i], s[i]) <= tol[2] and out_ok(out[r, :, i], o[:, i], np.array(sizes)[:, i], tol)
    rest = [i for i in range(slots) if i not in index.tolist()]
    assert torch.equal(pool[rest], before[rest])


def test_step_padding_and_doubled_entries():
    d, h = 64, 2
    x = draw(6, h, h, d, "f32", seed=11)
    pool = torch.randn(4, h, d, d, device=DEV)
    want_pool = pool.clone()
    vda = binding.Vda(d, "f32")
    some = torch.tensor([0, 2], device=DEV)
    want = vda.token_step(**{n: t[some].contiguous() for n, t in x.items()}, state=want_pool,
                          index=torch.tensor([3, 0], dtype=torch.int32, device=DEV))
    out = torch.full((6, h, d), 5.0, device=DEV)
    vda.token_step(**x, state=pool, index=torch.tensor([3, -1, 0, 4, -2147483648, 2147483647], dtype=torch.int32, device=DEV), out=out)
    torch.cuda.synchronize()
    assert vda.status() == binding.VDN_OK
    assert torch.equal(pool, want_pool) and torch.equal(out[some], want) and (out[[1, 3, 4, 5]] == 5).all()
    # the same state twice: the first entry has it, the second is left out and reported
    pool, out = want_pool.clone(), torch.full((2, h, d), 5.0, device=DEV)
    one = want_pool.clone()
    two = {n: t[:2].contiguous() for n, t in x.items()}
    want = vda.token_step(**{n: t[:1].contiguous() for n, t in x.items()}, state=one, index=torch.tensor([2], dtype=torch.int32, device=DEV))
    vda.token_step(**two, state=pool, index=torch.tensor([2, 2], dtype=torch.int32, device=DEV), out=out)
    torch.cuda.synchronize()
    assert vda.status() == binding.VDN_ERR_INVALID_ARG and vda.clear_status() == binding.VDN_ERR_INVALID_ARG
    assert vda.status() == binding.VDN_OK
    assert torch.equal(pool, one) and torch.equal(out[:1], want) and (out[1] == 5).all()


def test_step_captured_and_replayed():
    d, h = 128, 2
    x = draw(3, h, h, d, "bf16", seed=12)
    pool = torch.randn(3, h, d, d, device=DEV)
    index = torch.tensor([2, 0, 1], dtype=torch.int32, device=DEV)
    vda = binding.Vda(d, "bf16")
    want_pool = pool.clone()
    for _ in range(3):
        want = vda.token_step(**x, state=want_pool, index=index)
    vda.token_step(**x, state=pool.clone(), index=index)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = vda.token_step(**x, state=pool, index=index)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(pool, want_pool) and torch.equal(out, want)


# ------------------------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
def test_prompt_then_tokens_then_the_video_layer(dtype, d):
    """A prompt is scanned, a few tokens follow one by one, and the state is the text state of the video layer."""
    h, n, more = 2, 77, 3
    x = draw(n + more, h, h, d, dtype, seed=13)
    vda = binding.Vda(d, dtype)
    first = {m: t[:n].contiguous() for m, t in x.items()}
    out, state = vda.token_scan(**first)
    outs = [out]
    for t in range(n, n + more):
        outs.append(vda.token_step(**{m: y[t:t + 1].contiguous() for m, y in x.items()}, state=state))
    sizes = []
    want_o, want_s = tok.delta_rule(*(np64(x[m]) for m in ("q", "k", "v", "beta", "log_alpha")), sizes=sizes)
    tol = tolerances(dtype, d, n + more, tensor_cores(dtype, d))
    for i in range(h):
        assert rel(state[0, i], want_s[i]) <= tol[2]
        assert out_ok(torch.cat(outs)[:, i], want_o[:, i], np.array(sizes)[:, i], tol)
    w = inputs.VdaWorkload("joined", B=1, H=h, d=d, T=3, F=32, dtype=dtype, seed=4)
    y = inputs.generate(w, DEV)
    got = vda.forward(y["q"], y["k"], y["v"], y["beta"], y["gate"], s0=state)
    torch.cuda.synchronize()
    for i in range(h):
        ref = orc.vda_slice(*inputs.head_slice(y, 0, i), 1e-6, s0=want_s[i])["out"]
        assert orc.slice_error(np64(got[0, :, :, i]), ref) <= (1e-4 if dtype == "f32" else 2e-2)


# --------------------------------------------------------------------------------------------------------------- rotate
def rotate_case(dtype, d, B, T, Y, X, h, hk, half, norm, explicit, pairs, inverse=False, seed=0):
    g = torch.Generator().manual_seed(seed)
    q, k = (torch.randn(B, T, Y * X, n, d, generator=g).to(TYPES[dtype]).to(DEV) for n in (h, hk))
    t = pairs // 4
    y = (pairs - t) // 2
    freq, axis = binding.rotary_tables((t, y, pairs - t - y), theta=500.0)
    axis[pairs // 2] = 5                                         # one pair on no axis at all
    n = B * T * Y * X
    pos = torch.randint(-200000, 200000, (3, n), generator=g, dtype=torch.int32) if explicit else None
    wq, wk = ((1 + 0.2 * torch.randn(d, generator=g)).to(DEV) for _ in range(2)) if norm else (None, None)
    kw = dict(half=half, inverse=inverse, q_weight=wq, k_weight=wk, norm_eps=1e-5 if norm else 0.0)
    at = dict(positions=pos.to(DEV)) if explicit else dict(Y=Y, X=X, t0=11)
    vda = binding.Vda(d, dtype)
    got = vda.rotate(q, k, freq.to(DEV), axis.to(DEV), **at, **kw)
    torch.cuda.synchronize()
    where = pos.numpy() if explicit else tok.grid_positions(B, T, Y, X, 11)
    for x, y, w in ((q, got[0], wq), (k, got[1], wk)):
        want = tok.rotary(np64(x).reshape(n, -1, d), where, freq.tolist(), axis.tolist(), half, inverse, np64(w), kw["norm_eps"])
        # one rounding to io_dtype; in 32 bits: the angle's last fraction of a turn (2 pi 2^-25), the cosine's and sine's
        # 2^-23, three roundings of the rotation and six of the norm, each relative to the pair's size
        lead = float(np.abs(want).max())
        tol = (U32 if dtype == "f32" else U16) * np.abs(want) + (2 * np.pi / 2 + 2 + 3 + 6) * U32 * np.sqrt(2) * lead
        assert (np.abs(np64(y).reshape(n, -1, d) - want) <= tol).all()
    return q, k, freq.to(DEV), axis.to(DEV), at, kw, got, vda


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("norm,explicit", [(False, False), (True, True), (True, False), (False, True)])
def test_rotate(dtype, d, half, norm, explicit):
    for B, T, Y, X, h, hk, pairs in ((1, 1, 1, 1, 1, 1, d // 2), (2, 3, 5, 7, 4, 2, d // 2), (1, 2, 9, 11, 5, 1, d // 4),
                                     (1, 33, 6, 5, 3, 3, 24)):
        rotate_case(dtype, d, B, T, Y, X, h, hk, half, norm, explicit, pairs)
    if not half:
        rotate_case(dtype, d, 1, 2, 3, 3, 2, 2, half, norm, explicit, 21)     # an odd number of pairs, the rest passing through


def test_rotate_in_place_slices_queries_only_and_inverse():
    q, k, freq, axis, at, kw, got, vda = rotate_case("bf16", 128, 2, 3, 5, 7, 4, 2, True, False, False, 64)
    both = torch.cat([q, k, q], 3)
    a, b = both[..., :4, :], both[..., 4:6, :]
    vda.rotate(a, b, freq, axis, out=(a, b), **at, **kw)
    assert torch.equal(a, got[0]) and torch.equal(b, got[1]) and torch.equal(both[..., 6:, :], q)
    only, none = vda.rotate(q, None, freq, axis, **at, **kw)
    assert none is None and torch.equal(only, got[0])
    q, k, freq, axis, at, kw, got, vda = rotate_case("f32", 64, 1, 2, 3, 4, 2, 2, False, False, True, 32)
    kw["inverse"] = True
    back = vda.rotate(*got, freq, axis, **at, **kw)
    torch.cuda.synchronize()
    for x, y in zip((q, k), back):
        assert (x - y).abs().max() <= 2 * (2 * np.pi / 2 + 2 + 3) * U32 * 2 ** 0.5 * x.abs().max()


def test_rotate_inverse_is_the_gradient():
    """sum(w . rotate(x)) has the gradient rotate(w, inverse): against differences in the direction of one channel."""
    q, k, freq, axis, at, kw, got, vda = rotate_case("f32", 64, 1, 2, 2, 3, 1, 1, True, False, True, 32)
    w = torch.randn_like(q)
    grad = vda.rotate(w, None, freq, axis, **at, **dict(kw, inverse=True))[0]
    for c in (0, 7, 40):
        step = torch.zeros_like(q)
        step[0, 1, 3, 0, c] = 0.5
        up, down = (vda.rotate(q + s * step, None, freq, axis, **at, **kw)[0] for s in (1, -1))
        slope = float((w.double() * (up.double() - down.double())).sum())
        assert abs(slope - float(grad[0, 1, 3, 0, c])) <= 64 * 2 * 8 * U32 * float(w.abs().max() * q.abs().max() * 2)


def test_rotate_on_another_stream_and_captured():
    q, k, freq, axis, at, kw, got, vda = rotate_case("bf16", 128, 1, 4, 6, 6, 4, 4, False, True, False, 64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = vda.rotate(q, k, freq, axis, **at, **kw, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(other[0], got[0]) and torch.equal(other[1], got[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kept = vda.rotate(q, k, freq, axis, **at, **kw)
    q.mul_(2)
    g.replay()
    torch.cuda.synchronize()
    again = vda.rotate(q, k, freq, axis, **at, **kw)
    assert torch.equal(kept[0], again[0]) and torch.equal(kept[1], again[1])


# -------------------------------------------------------------------------------------------------------------- refusals
def test_refusals_with_a_handle():
    d, h = 64, 2
    vda = binding.Vda(d, "f32")
    x = draw(4, h, h, d, "f32")
    cu = torch.tensor([0, 2, 4], dtype=torch.int32, device=DEV)
    state = torch.zeros(2, h, d, d, device=DEV)
    with pytest.raises(ValueError, match="cu_seqlens"):
        vda.token_scan(**x, cu_seqlens=cu.long())
    with pytest.raises(ValueError, match="cu_seqlens"):
        vda.token_scan(**x, cu_seqlens=cu[:1])
    with pytest.raises(ValueError, match="s0"):
        vda.token_scan(**x, cu_seqlens=cu, s0=state[:1])
    with pytest.raises(ValueError, match="state"):
        vda.token_scan(**x, cu_seqlens=cu, state=state.double())
    with pytest.raises(ValueError, match="q"):
        vda.token_scan(**dict(x, q=x["q"].cpu()))
    for kw in (dict(scale=float("nan")), dict(l2_eps=-1.0), dict(l2_eps=float("inf")), dict(out=x["v"])):
        with pytest.raises(binding.VdnError, match="INVALID_ARG"):
            vda.token_scan(**x, **kw)
    with pytest.raises(ValueError, match="index"):
        vda.token_step(**x, state=state, index=cu)
    with pytest.raises(ValueError, match="state"):
        vda.token_step(**x, state=None)
    with pytest.raises(binding.VdnError, match="INVALID_ARG"):
        vda.token_step(**x, state=state)                              # four requests, two states, no index
    q = torch.zeros(1, 2, 6, h, d, device=DEV)
    freq, axis = (t.to(DEV) for t in binding.rotary_tables((8, 8, 8)))
    for kw in (dict(Y=2, X=2), dict(Y=-2, X=-3), dict(Y=2, X=3, norm_eps=1e-6, inverse=True), dict(Y=2, X=3, q_weight=torch.ones(d, device=DEV)),
               dict(Y=2, X=3, norm_eps=float("nan")), dict(Y=2, X=3, t0=2 ** 31 - 1)):
        with pytest.raises(binding.VdnError, match="INVALID_ARG"):
            vda.rotate(q, None, freq, axis, **kw)
    with pytest.raises(binding.VdnError, match="multiple of 8"):
        vda.rotate(q, None, freq[:20].contiguous(), axis[:20].contiguous(), Y=2, X=3, half=True)
    with pytest.raises(binding.VdnError, match="pairs"):
        vda.rotate(q, None, freq.repeat(2), axis.repeat(2), Y=2, X=3)
    for kw in (dict(), dict(positions=torch.zeros(3, 5, dtype=torch.int32, device=DEV)), dict(Y=2, X=3, out=(q[:, :1], None))):
        with pytest.raises(ValueError):
            vda.rotate(q, None, freq, axis, **kw)
    assert vda.status() == binding.VDN_OK
