"""rotate against its 64-bit statement where a block of threads covers several tokens (8 * 148 tokens and more)."""
import numpy as np
import pytest
import torch

from oracle import token_oracle as tok
from paper_2609_20744_b200 import binding, build

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U16, U32 = 2.0 ** -8, 2.0 ** -24        # half a step of bf16 and of fp32


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.load_library()


def allowed(dtype, want):
    """One rounding to io_dtype; in 32 bits the angle's last fraction of a turn (2 pi 2^-25), the cosine's and sine's 2^-23, three
    roundings of the rotation and six of the norm, each relative to the pair's size."""
    return (U32 if dtype == "f32" else U16) * np.abs(want) + (np.pi + 2 + 3 + 6) * U32 * np.sqrt(2) * np.abs(want).max()


# 2511 and 2701 tokens: tiles of up to 4; 19277: of up to 32, the last of 13
@pytest.mark.parametrize("B,T,Y,X,h,hk", [(*shape, *heads) for shape in ((1, 27, 3, 31), (1, 37, 1, 73), (1, 37, 521, 1))
                                          for heads in ((1, None), (1, 1), (3, None), (5, 2), (3, 2), (5, 1))] + [(1, 27, 3, 31, 40, 40)])
@pytest.mark.parametrize("dtype,d,half,norm", [("f32", 64, False, False), ("f32", 64, True, True), ("f32", 128, True, False),
                                               ("bf16", 64, False, True), ("bf16", 128, True, True), ("bf16", 128, False, False)])
def test_tiles_of_several_tokens(dtype, d, half, norm, B, T, Y, X, h, hk):
    n = B * T * Y * X
    g = torch.Generator().manual_seed(n + h)
    q, k = (None if m is None else torch.randn(B, T, Y * X, m, d, generator=g).to(TYPES[dtype]).to(DEV) for m in (h, hk))
    pairs = d // 2 - 8
    freq, axis = binding.rotary_tables((pairs // 4, pairs // 4, pairs - pairs // 2), theta=500.0)
    wq, wk = ((1 + 0.2 * torch.randn(d, generator=g)).to(DEV) for _ in range(2)) if norm else (None, None)
    vda = binding.Vda(d, dtype)
    got = vda.rotate(q, k, freq.to(DEV), axis.to(DEV), Y=Y, X=X, t0=11, half=half, q_weight=wq, k_weight=wk if k is not None else None,
                     norm_eps=1e-5 if norm else 0.0)
    torch.cuda.synchronize()
    assert vda.status() == binding.VDN_OK
    where = tok.grid_positions(B, T, Y, X, 11)
    for x, y, w in ((q, got[0], wq), (k, got[1], wk)):
        if x is None:
            assert y is None
            continue
        want = tok.rotary(x.double().cpu().numpy().reshape(n, -1, d), where, freq.tolist(), axis.tolist(), half,
                          weight=None if w is None else w.double().cpu().numpy(), norm_eps=1e-5 if norm else 0.0)
        assert (np.abs(y.double().cpu().numpy().reshape(n, -1, d) - want) <= allowed(dtype, want)).all()


def test_one_head_of_a_wider_tensor():
    """Queries of one head alone, each token's row inside a wider one: what lies beside stays."""
    n, d = 5000, 128
    wide = torch.randn(1, 1, n, 3, d, device=DEV).bfloat16()
    before = wide.clone()
    freq, axis = (t.to(DEV) for t in binding.rotary_tables((16, 24, 24)))
    vda = binding.Vda(d, "bf16")
    want, _ = vda.rotate(before[..., 1:2, :].contiguous(), None, freq, axis, Y=50, X=100)
    mid = wide[..., 1:2, :]
    vda.rotate(mid, None, freq, axis, Y=50, X=100, out=(mid, None))
    torch.cuda.synchronize()
    assert torch.equal(wide[..., 1:2, :], want) and torch.equal(wide[..., ::2, :], before[..., ::2, :])
    ref = tok.rotary(before[..., 1:2, :].double().cpu().numpy().reshape(n, 1, d), tok.grid_positions(1, 1, 50, 100), freq.tolist(),
                     axis.tolist())
    assert (np.abs(want.double().cpu().numpy().reshape(n, 1, d) - ref) <= allowed("bf16", ref)).all()


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("half,pairs", [(False, 21), (False, 32), (True, 24), (True, 32)])
@pytest.mark.parametrize("frames", [1, 40])
def test_channels_that_are_not_turned_are_copied(dtype, d, half, pairs, frames):
    """Channels beyond the pairs and a pair on no axis: infinities, NaN and signed zeros beside one another stay what they are, and
    the turned channels are what they are without them."""
    T, F, h = frames, 64, 3
    g = torch.Generator().manual_seed(d + pairs)
    freq, axis = binding.rotary_tables((pairs // 4, pairs // 4, pairs - 2 * (pairs // 4)), theta=500.0)
    off = [3, pairs - 1]
    axis[3], axis[pairs - 1] = -1, 7
    turned = torch.zeros(d, dtype=torch.bool)
    for p in range(pairs):
        if p not in off:
            turned[[p, p + pairs] if half else [2 * p, 2 * p + 1]] = True
    kept = (~turned).nonzero()[:, 0]
    clean = torch.randn(1, T, F, h, d, generator=g)
    x = clean.clone()
    odd = torch.tensor([float("inf"), -0.0, float("nan"), 1.5, -float("inf"), 0.0, 2.5, -0.0])
    which = torch.randint(0, 8, x[..., kept].shape, generator=g)
    x[..., kept] = odd[which]
    x, clean = (t.to(TYPES[dtype]).to(DEV) for t in (x, clean))
    vda = binding.Vda(d, dtype)
    at = dict(freq=freq.to(DEV), axis=axis.to(DEV), Y=8, X=8, half=half)
    got, _ = vda.rotate(x, None, **at)
    want, _ = vda.rotate(clean, None, **at)
    assert torch.equal(got[..., turned.to(DEV)], want[..., turned.to(DEV)])
    got, x = got[..., kept.to(DEV)], x[..., kept.to(DEV)]
    nan = x.isnan()
    bits = torch.int32 if dtype == "f32" else torch.int16
    assert torch.equal(got.isnan(), nan) and torch.equal(got[~nan].view(bits), x[~nan].view(bits))


@pytest.mark.parametrize("dtype,d,half", [("f32", 64, True), ("bf16", 128, False)])
@pytest.mark.parametrize("h,hk", [(1, None), (4, 2)])
def test_given_positions_in_tiles_of_several_tokens(dtype, d, half, h, hk):
    """Two clips of 1571 tokens, any positions, one pair on no axis, turned and turned back."""
    B, T, F = 2, 1571, 1
    n = B * T * F
    g = torch.Generator().manual_seed(h)
    q, k = (None if m is None else torch.randn(B, T, F, m, d, generator=g).to(TYPES[dtype]).to(DEV) for m in (h, hk))
    freq, axis = binding.rotary_tables((8, 8, 8), theta=500.0)
    axis[9] = 3
    pos = torch.randint(-200000, 200000, (3, n), generator=g, dtype=torch.int32)
    vda = binding.Vda(d, dtype)
    for inverse in (False, True):
        got = vda.rotate(q, k, freq.to(DEV), axis.to(DEV), positions=pos.to(DEV), half=half, inverse=inverse)
        for x, y in zip((q, k), got):
            if x is None:
                continue
            want = tok.rotary(x.double().cpu().numpy().reshape(n, -1, d), pos.numpy(), freq.tolist(), axis.tolist(), half, inverse)
            assert (np.abs(y.double().cpu().numpy().reshape(n, -1, d) - want) <= allowed(dtype, want)).all()
