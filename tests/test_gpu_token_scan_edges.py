"""token_scan where its decays, its cuts and its inputs are at their edges, against the 64-bit statement of tests/test_gpu_token_ops.py's
tolerances."""
import numpy as np
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
