"""token_scan where its decays, its cuts and its inputs are at their edges, against the 64-bit statement of tests/test_gpu_token_ops.py's
tolerances."""
import ctypes

import pytest
import torch

from oracle import token_oracle as tok
from paper_2609_20744_b200 import binding, build
from tests.test_gpu_token_ops import DEV, check_scan, draw, np64, rel, tolerances

pytestmark = pytest.mark.gpu
CHUNKS = ["token_prep", "token_chain"]
PARTS = ["token_prep", "token_compose", "token_join", "token_chain"]


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.load_library()


def kernels(vda):
    return [k[0] for k in vda.kernel_times()]


@pytest.mark.parametrize("l2", [False, True])
@pytest.mark.parametrize("pattern", ["resets, then two", "every other", "every fourth", "strong", "resets, then slow"])
def test_state_after_strong_decays(pattern, l2):
    """Many resets or strong decays among 16 tokens, slow decay after them: the state hangs on the few tokens since, whose factors
    e^{G_i - G_j} are then differences of large sums.  One key and beta = 1: each token's difference from the one before is
    multiplied by such a factor.  Every factor has 16 bits (2^-16 relative), the bound of tolerances() for few tokens: what came
    before the last reset rounds to nothing."""
    d, h, lens = 128, 8, [128, 144, 190, 96, 161, 64, 207, 80]
    n = sum(lens)
    g = torch.Generator().manual_seed(7)
    x = draw(n, h, h, d, "bf16", seed=21, l2=l2)
    x["k"][:] = x["k"][:1].clone()
    x["beta"][:] = 1
    la = -0.01 * (1 + torch.rand(n, h, generator=g))
    at = 0
    for m in lens:
        back = torch.arange(m).flip(0)                    # tokens to the end of the sequence
        here = la[at:at + m]
        if pattern == "resets, then two":
            here[back >= 2] = -float("inf")
        elif pattern == "every other":
            here[back % 2 == 1] = -float("inf")
        elif pattern == "every fourth":
            here[back % 4 == 3] = -float("inf")
        elif pattern == "strong":
            here[back >= 3] = -50 * torch.rand(int((back >= 3).sum()), h, generator=g)
        else:
            here[(back >= 7) & (back < 15)] = -float("inf")
        at += m
    x["log_alpha"] = la.to(DEV)
    cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32).to(DEV)
    eps = 1e-6 if l2 else 0.0
    vda = binding.Vda(d, "bf16")
    vda.profile(True)
    out, state = vda.token_scan(**x, cu_seqlens=cu, l2_eps=eps)
    assert kernels(vda) == CHUNKS
    _, want = tok.packed(*(np64(x[m]) for m in ("q", "k", "v", "beta")), lens, np64(x["log_alpha"]), None, 1.0, eps)
    limit = tolerances("bf16", d, 16, True)[2]
    worst = max(rel(state[i, j], want[i, j]) for i in range(len(lens)) for j in range(h))
    assert worst <= limit, (worst, limit)


def spoil(x, name, t, value):
    """The inputs with token t of one of them set to `value` (q, k: all heads; v: one channel; gates: one head)."""
    x = dict(x, **{name: x[name].clone()})
    if name == "v":
        x[name][t, :, 5] = value
    elif name in ("q", "k"):
        x[name][t] = value
    else:
        x[name][t, 0] = value
    return x


@pytest.mark.parametrize("dtype,d,flags", [("f32", 64, 0), ("f32", 128, 0), ("bf16", 64, 0),
                                           ("bf16", 128, binding.VDN_FLAG_FORCE_SIMT)])
@pytest.mark.parametrize("n,names", [(7, ["token_few"]), (103, ["token_coef", "token_walk"]),
                                     (2000, ["token_coef", "token_walk_compose", "token_join", "token_walk"])])
def test_plain_kernels_keep_what_is_not_finite_from_the_tokens_before(dtype, d, flags, n, names):
    """Token by token or four at a step, whole or in parts: token t reaches itself and what follows, a value only its own channel."""
    h = 2
    x = draw(n, h, h, d, dtype, seed=22)
    vda = binding.Vda(d, dtype, flags=flags)
    vda.profile(True)
    clean, state = vda.token_scan(**x)
    assert kernels(vda) == names
    for t in (n - 2, n - 3, n - 4, n - 5, n // 2):
        for name, value in (("q", float("nan")), ("k", float("inf")), ("v", float("nan")), ("v", float("inf")), ("beta", float("nan")),
                            ("log_alpha", float("nan"))):
            out, after = vda.token_scan(**spoil(x, name, t, value))
            assert torch.equal(out[:t], clean[:t]), (name, t)
            if name == "q":
                assert torch.equal(out[t + 1:], clean[t + 1:]) and torch.equal(after, state) and out[t].isnan().all()
            elif name == "v":
                other = torch.arange(d, device=DEV) != 5
                assert torch.equal(out[..., other], clean[..., other]) and torch.equal(after[:, :, other], state[:, :, other])
                assert not out[t:, :, 5].isfinite().any()


def test_chunks_keep_what_is_not_finite_from_the_chunks_before():
    """In chunks of 64 such a value reaches its whole chunk and what follows, but no chunk before, and a value only its own channel."""
    d, h = 128, 2
    for n, t in ((300, 150), (5000, 4100)):
        x = draw(n, h, h, d, "bf16", seed=23)
        vda = binding.Vda(d, "bf16")
        vda.profile(True)
        clean, state = vda.token_scan(**x)
        assert kernels(vda) == (CHUNKS if n == 300 else PARTS)
        first = t // 64 * 64
        for name in ("q", "k", "v", "beta", "log_alpha"):
            out, after = vda.token_scan(**spoil(x, name, t, float("nan")))
            assert torch.equal(out[:first], clean[:first]), name
            if name == "q":
                assert torch.equal(out[t + 1:], clean[t + 1:]) and torch.equal(out[first:t], clean[first:t]) and torch.equal(after, state)
            elif name == "v":
                other = torch.arange(d, device=DEV) != 5
                assert torch.equal(out[..., other], clean[..., other]) and torch.equal(after[:, :, other], state[:, :, other])


def in_chunks(q, k, v, beta, log_alpha, s0, scale, l2_eps, state_tol, C=64):
    """One sequence in 64 bits, chunk by chunk, and how far the tensor cores may be off.  q, k, v [n, H, d], gates [n, H], s0 [H, d, d];
    returns read-out [n, H, d], its bound without the last rounding, state.

    O = e^G S q + P X with P = M T, M the decayed q.k, T the inverse of I + L.  Every factor but q and k has two bf16 parts, off by
    2^-16 (r, e^G: 2^-20), and accumulators are fp32: the result is off by 2^-16 of each of S, X, M, T and P's terms, taken without
    their signs, and by what the state is off, state_tol of its norm (and of X's, which has it as e^G S k)."""
    q, k, v, beta = (t.double() for t in (q, k, v, beta))
    g = log_alpha.double().clamp(min=-104) if log_alpha is not None else torch.zeros_like(beta)
    if l2_eps > 0:
        q, k = (t / torch.sqrt((t * t).sum(-1, keepdim=True) + l2_eps) for t in (q, k))
    n, h, d = v.shape
    r = h // q.shape[1]
    q, k = q.repeat_interleave(r, 1), k.repeat_interleave(r, 1)
    S = s0.double().clone() if s0 is not None else torch.zeros(h, d, d, dtype=torch.float64, device=v.device)
    want, off = torch.empty_like(v), torch.empty_like(v)
    for c in range(0, n, C):
        w = slice(c, min(n, c + C))
        Q, K, V = (t[w].transpose(0, 1) for t in (q, k, v))                # [H, C, d]
        b, G = beta[w].T, g[w].T.cumsum(-1)
        decay = torch.exp((G[:, :, None] - G[:, None]).tril()).tril()
        eye = torch.eye(G.shape[1], dtype=torch.float64, device=v.device)
        T = torch.linalg.inv(eye + (b[:, :, None] * decay * (K @ K.mT)).tril(-1)) * b[:, None]
        M, e = decay * (Q @ K.mT), torch.exp(G)[..., None]
        X = V - e * (K @ S.mT)
        P = M.abs() @ T.abs()
        norm = S.flatten(1).norm(dim=1)[:, None, None] * state_tol / d ** 0.5
        from_state = norm * (e * Q.norm(dim=2, keepdim=True) + P @ (e * K.norm(dim=2, keepdim=True)))
        want[w] = (scale * (e * (Q @ S.mT) + M @ T @ X)).transpose(0, 1)
        off[w] = (abs(scale) * (2.0 ** -16 * (e * (Q.abs() @ S.abs().mT) + 4 * (P @ X.abs())) + from_state)).transpose(0, 1)
        S = torch.exp(G[:, -1])[:, None, None] * S + (T @ X).mT @ (torch.exp(G[:, -1:] - G)[..., None] * K)
    return want, off, S


def check_chunks(vda, x, lens, names, s0=None, in_place=False, scale=0.5, l2_eps=0.0, walks=1):
    """token_scan on the tensor cores against in_chunks, sequence by sequence and head by head."""
    d = 128
    cu = torch.tensor([0] + list(lens)).cumsum(0).to(torch.int32).to(DEV)
    first = s0.clone() if s0 is not None else None
    vda.profile(True)
    out, state = vda.token_scan(**x, cu_seqlens=cu, s0=s0, state=s0 if in_place else None, scale=scale, l2_eps=l2_eps)
    torch.cuda.synchronize()
    assert vda.status() == binding.VDN_OK and kernels(vda) == names
    at = 0
    for i, n in enumerate(lens):
        w = slice(at, at + n)
        tol = walks * tolerances("bf16", d, n, True)[2]
        want, off, want_s = in_chunks(*(x[m][w] if x[m] is not None else None for m in ("q", "k", "v", "beta", "log_alpha")),
                                      first[i] if first is not None else None, scale, l2_eps, tol)
        for j in range(state.shape[1]):
            assert float((state[i, j].double() - want_s[j]).norm()) <= tol * float(want_s[j].norm()), (i, j, n)
            far = float((out[w, j].double() - want[:, j]).norm())
            assert far <= 2.0 ** -8 * float(want[:, j].norm()) + float(off[:, j].norm()), (i, j, n)
        at += n


@pytest.mark.parametrize("lens,h,hk,l2,decay,first", [
    ([131, 0, 3003, 64, 2500], 4, 2, 1e-6, True, True), ([1500, 1501], 4, 4, 0.0, False, True), ([1, 5000, 3], 1, 1, 1e-6, True, False),
    ([2049], 6, 2, 0.0, True, True), ([100, 4000], 9, 3, 1e-6, False, False)], ids=str)
def test_cut_sequences(lens, h, hk, l2, decay, first):
    """Sequences in parts that start anywhere, several in a call, with shared key heads, normalised keys, resets inside a part and at its
    border, states in place.  A part's last state is enter M + J: M, J and the walk itself are each off as a whole sequence's state
    is, hence three times its tolerance."""
    d, n = 128, sum(lens)
    x = draw(n, h, hk, d, "bf16", seed=31, l2=l2 > 0, decay=decay)
    if decay:
        at = max(range(len(lens)), key=lambda i: lens[i])
        start = sum(lens[:at])
        x["log_alpha"][[start + 700, start + 1024, start + lens[at] - 30]] = -float("inf")
    g = torch.Generator().manual_seed(32)
    s0 = 0.3 * torch.randn(len(lens), h, d, d, generator=g).to(DEV) if first else None
    check_chunks(binding.Vda(d, "bf16"), x, lens, PARTS, s0, first, l2_eps=l2, walks=3)


@pytest.mark.parametrize("seqs,h,hk", [(90, 6, 2), (256, 4, 4), (300, 8, 4)])
def test_many_sequences_in_chunks(seqs, h, hk):
    """More chains than SMs: the longest first up to 256 sequences, as they come beyond."""
    d = 128
    g = torch.Generator().manual_seed(seqs)
    lens = torch.randint(0, 170, (seqs,), generator=g).tolist()
    x = draw(sum(lens), h, hk, d, "bf16", seed=33, l2=True)
    s0 = 0.3 * torch.randn(seqs, h, d, d, generator=g).to(DEV)
    check_chunks(binding.Vda(d, "bf16"), x, lens, CHUNKS, s0, True, l2_eps=1e-6)


def test_uneven_lengths_in_chunks():
    lens = [5, 0, 64, 1, 130, 0, 63, 700, 2, 129]
    for h, hk, l2, decay in ((3, 3, 0.0, True), (4, 1, 1e-6, True), (4, 2, 0.0, False)):
        x = draw(sum(lens), h, hk, 128, "bf16", seed=34, l2=l2 > 0, decay=decay)
        check_chunks(binding.Vda(128, "bf16"), x, lens, CHUNKS, l2_eps=l2)


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
@pytest.mark.parametrize("n", [5, 40, 300])
def test_keys_of_zero_with_the_smallest_eps(dtype, d, n):
    """1 / l2_eps is the factor between two keys of zero: finite down to the smallest eps that is taken, and nothing is written."""
    x = draw(n, 2, 2, d, dtype, seed=41)
    x["k"][n // 3:] = 0
    x["q"][n // 2:] = 0
    vda = binding.Vda(d, dtype)
    out, state = vda.token_scan(**x, l2_eps=1.2e-38)
    assert out.isfinite().all() and state.isfinite().all() and (out[n // 2:] == 0).all()
    step = {m: t[-3:] for m, t in x.items()}
    pool = torch.randn(3, 2, d, d, device=DEV)
    want = pool * torch.exp(step["log_alpha"])[..., None, None]
    assert (vda.token_step(**step, state=pool, l2_eps=1.2e-38) == 0).all()
    assert float((pool - want).norm()) <= 2.0 ** -22 * float(want.norm())
    for eps in (1e-38, 1e-40, 1e-45):
        with pytest.raises(binding.VdnError, match="l2_eps"):
            vda.token_scan(**x, l2_eps=eps)
        with pytest.raises(binding.VdnError, match="l2_eps"):
            vda.token_step(**step, state=pool, l2_eps=eps)


@pytest.mark.parametrize("dtype,d,flags", [("f32", 64, 0), ("f32", 128, 0), ("bf16", 64, 0), ("bf16", 128, 0),
                                           ("bf16", 128, binding.VDN_FLAG_FORCE_SIMT)])
@pytest.mark.parametrize("gate", [-1e-4, -1e-6, -1e-7, -4e-8, -2e-8, -0.02, -0.5, 0.0])
def test_constant_gates_near_one(dtype, d, flags, gate):
    """A gate that is the same for every token and head: what rounding does to it must not add up over the tokens.  A state's element is
    rounded at most five times in four tokens, and what is written (a 1/sqrt(d)-th of the state or so) by its dot product: three
    halves of a step a token, independent, 3 sqrt(n) u32; on the tensor cores 4 * 2^-16 besides."""
    n, h = 3000, 4
    x = draw(n, h, h, d, dtype, seed=42, decay=False)
    x["log_alpha"] = torch.full((n, h), gate, device=DEV)
    tol = 3 * n ** 0.5 * 2.0 ** -24
    vda = binding.Vda(d, dtype, flags=flags)
    vda.profile(True)
    _, state = vda.token_scan(**x)
    chunks = "token_chain" in kernels(vda)
    want = in_chunks(*(x[m] for m in ("q", "k", "v", "beta", "log_alpha")), None, 1.0, 0.0, tol)[2]
    far = (state[0].double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)
    assert float(far.max()) <= tol + (4 * 2.0 ** -16 if chunks else 0)
    # as one request of as many tokens
    pool = torch.zeros(1, h, d, d, device=DEV)
    vda.token_step(**{m: t[None] for m, t in x.items()}, state=pool)
    far = (pool[0].double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)
    assert float(far.max()) <= tol


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("f32", 128), ("bf16", 128)])
def test_a_long_sequence_among_single_tokens(dtype, d):
    """Few tokens a sequence on average: each sequence goes token by token, the long one too."""
    lens = [1] * 150 + [700] + [1, 0, 2] * 20
    x = draw(sum(lens), 2, 1, d, dtype, seed=43)
    s0 = 0.3 * torch.randn(len(lens), 2, d, d, generator=torch.Generator().manual_seed(44)).to(DEV)
    vda = binding.Vda(d, dtype)
    vda.profile(True)
    check_scan(vda, x, lens, dtype, d, False, s0, scale=0.5)
    assert kernels(vda) == ["token_few"]


@pytest.mark.parametrize("n", [5, 40, 300, 3000])
@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
def test_a_state_that_nobody_wants(dtype, d, n):
    """The C entry point takes NULL for the last states: the read-outs are the same."""
    x = draw(n, 2, 2, d, dtype, seed=45)
    s0 = torch.randn(1, 2, d, d, device=DEV)
    vda = binding.Vda(d, dtype)
    want, _ = vda.token_scan(**x, s0=s0)
    prm = binding.VdnTokenParams(ctypes.sizeof(binding.VdnTokenParams), 2, 2, 1, 1.0, 0.0, None, None, x["log_alpha"].data_ptr(),
                                 s0.data_ptr(), None)
    need = vda.lib.vdn_vda_token_scan_workspace_bytes(vda.h, n, ctypes.byref(prm))
    ws, out = torch.empty(need, dtype=torch.uint8, device=DEV), torch.empty_like(x["v"])
    stream = torch.cuda.current_stream().cuda_stream
    args = (vda.h, x["q"].data_ptr(), x["k"].data_ptr(), x["v"].data_ptr(), x["beta"].data_ptr(), out.data_ptr(), n, ctypes.byref(prm))
    assert vda.lib.vdn_vda_token_scan(*args, ws.data_ptr() if need else None, need, stream) == binding.VDN_OK
    torch.cuda.synchronize()
    assert vda.status() == binding.VDN_OK and torch.equal(out, want)
    if need:
        assert binding.STATUS_NAMES[vda.lib.vdn_vda_token_scan(*args, ws.data_ptr(), need - 1, stream)] == "VDN_ERR_WORKSPACE"
