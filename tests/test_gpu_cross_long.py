"""cross_attention over so many keys that their sums are moved on the way: more than 256 tiles of 128 keys to one run of a kernel, which
takes many rows (few rows are cut into shorter parts).

Tolerances.  u32 = 2^-24.  The tensor cores add 16 keys at a time and cut off (2 u32), at most 2048 times before a sum moves on.  A sum of
weights has at most 8192 additions before it moves, each off by u32 either way: 8 sqrt(8192) u32 = 724 u32 is more than any will show.
Sums that moved are added in fp32, one for 32768 keys.  lse: off = (2 d + 12) u32 spread + 2^-21 + (724 + n / 32768) u32, and 4 u32 |lse|;
out: u |out| + (2 off + 2 * 2048 u32 + 2^-8 for weights in bf16) of sum_j p_j |v_j|.
"""
import math

import pytest
import torch

from paper_2609_20744_b200 import binding, build

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U32 = 2.0 ** -24
ROWS = 76 * 256                                                           # more than half as many tiles as SMs: the keys are not cut


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.load_library()


def check(vda, x, d, keys_of, picks):
    """Rows `picks` (batch row, query, head) against 64 bits; keys_of(b) gives (slice of k and v as rows, which count or None)."""
    out, lse = vda.cross_attention(**x, lse=True)
    torch.cuda.synchronize()
    assert vda.status() == binding.VDN_OK
    k, v = x["k"].reshape(-1, *x["k"].shape[-2:]), x["v"].reshape(-1, *x["v"].shape[-2:])
    group = x["q"].shape[-2] // k.shape[-2]
    for b, i, h in picks:
        at, on = keys_of(b)
        kk, vv = k[at, h // group].double(), v[at, h // group].double()
        if on is not None:
            kk, vv = kk[on], vv[on]
        n = kk.shape[0]
        got, got_lse = out[b, i, h].double(), float(lse[b, i, h])
        if n == 0:
            assert (got == 0).all() and got_lse == -math.inf
            continue
        q = x["q"][b, i, h].double()
        z = kk @ q * d ** -0.5
        want_lse = float(torch.logsumexp(z, 0))
        p = torch.exp(z - want_lse)
        want, weight = p @ vv, p @ vv.abs()
        spread = float((kk.abs() @ q.abs()).max()) * d ** -0.5
        off = (2 * d + 12) * U32 * spread + 2.0 ** -21 + (724 + n / 32768) * U32
        assert abs(got_lse - want_lse) <= off + 4 * U32 * abs(want_lse), (b, i, h, got_lse - want_lse)
        bound = 2.0 ** -8 * want.abs() + (2 * off + 2 * 2048 * U32 + 2.0 ** -8) * weight
        assert bool(((got - want).abs() <= bound).all()), (b, i, h, float(((got - want).abs() / bound).max()))
    return out, lse


@pytest.mark.parametrize("d", [64, 128])
def test_mean_of_ones_over_a_million_keys(d):
    """The weights of a row add up to one: all that is lost on the way shows.  What is allowed, 2 * 2048 u32 = 2.4e-4 and the mean of 2^20
    roundings of weights, is less than half a step below one (2^-9)."""
    n = 1 << 20
    g = torch.Generator(device=DEV).manual_seed(d)
    q = torch.randn(1, ROWS, 1, d, generator=g, device=DEV, dtype=torch.bfloat16)
    k = torch.randn(1, n, 1, d, generator=g, device=DEV, dtype=torch.bfloat16)
    vda = binding.Vda(d, "bf16")
    out, lse = vda.cross_attention(q, k, torch.ones_like(k), lse=True)
    assert vda.launch_count() == 1
    assert (out == 1).all(), float(out.float().mean())
    assert lse.isfinite().all() and vda.status() == binding.VDN_OK


@pytest.mark.parametrize("d", [64, 128])
def test_mean_of_ones_over_a_million_keys_in_f32(d):
    """Sum and weighted values take 64 + n / 64 additions, each off by at most u32 of a sum that grows to its end: u32 / 3 for each in the
    mean square, 8 sqrt(64 + n / 64) sqrt(2) u32 / 3 < 8 sqrt(64 + n / 64) u32 / 2 between the two."""
    n = 1 << 20
    g = torch.Generator(device=DEV).manual_seed(d)
    q = torch.randn(1, 128 * 148, 1, d, generator=g, device=DEV)
    k = torch.randn(1, n, 1, d, generator=g, device=DEV)
    vda = binding.Vda(d, "f32")
    out, lse = vda.cross_attention(q, k, torch.ones_like(k), lse=True)
    assert vda.launch_count() == 1
    assert float((out - 1).abs().max()) <= 8 * math.sqrt(64 + n / 64) * U32 / 2
    for i in range(0, q.shape[1], 2377):
        want = torch.logsumexp(k[0, :, 0].double() @ q[0, i, 0].double() * d ** -0.5, 0)
        assert abs(float(lse[0, i, 0]) - float(want)) <= 2.0 ** -18                        # 2 d u32 of a score of about 10, and the above


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [32768, 32769, 65536, 70001])
@pytest.mark.parametrize("louder", [False, True])
def test_keys_around_where_sums_move(d, n, louder):
    """Heads of a group; with `louder` keys that grow along the way, so that the maximum moves after the sums have."""
    g = torch.Generator(device=DEV).manual_seed(n + d)
    lq = ROWS // 2 + 77
    q = torch.randn(1, lq, 2, d, generator=g, device=DEV, dtype=torch.bfloat16)
    k = torch.randn(1, n, 1, d, generator=g, device=DEV)
    if louder:
        k *= torch.linspace(0.1, 4, n, device=DEV)[None, :, None, None]
    k = k.bfloat16()
    v = (torch.rand(1, n, 1, d, generator=g, device=DEV) + 0.25 * torch.randn(1, n, 1, d, generator=g, device=DEV)).bfloat16()
    vda = binding.Vda(d, "bf16")
    picks = [(0, i, h) for i in (0, 1, 127, 128, 255, lq // 2, lq - 78, lq - 1) for h in (0, 1)]
    check(vda, dict(q=q, k=k, v=v), d, lambda b: (slice(0, n), None), picks)
    assert vda.launch_count() == 1


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("packed", [False, True])
def test_one_long_encoder_among_short_ones(d, packed):
    """Batch rows one after another in a CTA, with sums that move and without, some without keys, long runs of masked ones (NaN in them)."""
    g = torch.Generator(device=DEV).manual_seed(d)
    lens = [0, 70000, 5, 40000, 130, 33000] + [100] * 34 if packed else [0, 50000, 5, 40000, 130, 33000, 49999, 32768] * 5
    B, lq, most = len(lens), 300, max(lens)
    lead = (sum(lens),) if packed else (B, most)
    q = torch.randn(B, lq, 2, d, generator=g, device=DEV, dtype=torch.bfloat16)
    k = torch.randn(*lead, 1, d, generator=g, device=DEV, dtype=torch.bfloat16)
    v = torch.rand(*lead, 1, d, generator=g, device=DEV).bfloat16()
    mask = torch.rand(*lead, generator=g, device=DEV) < 0.7
    first = [sum(lens[:b]) if packed else b * most for b in range(B)]
    flat = mask.view(-1)
    flat[first[1]: first[1] + 34000] = False
    flat[first[3] + 34000: first[3] + lens[3]] = False
    k[~mask], v[~mask] = float("nan"), float("nan")
    x = dict(q=q, k=k, v=v, mask=mask)
    if packed:
        x["cu_seqlens"] = torch.tensor([0] + lens).cumsum(0).to(torch.int32).to(DEV)
    else:
        x["lengths"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    at = lambda b: slice(first[b], first[b] + lens[b])  # noqa: E731
    picks = [(b, i, h) for b in (*range(8), B - 1) for i in (0, 150, lq - 1) for h in (0, 1)]
    vda = binding.Vda(d, "bf16")
    want = check(vda, x, d, lambda b: (at(b), flat[at(b)]), picks)
    # once more, captured, while another call runs on a stream of its own
    g1, side, other = torch.cuda.CUDAGraph(), torch.cuda.Stream(), binding.Vda(d, "bf16")
    torch.cuda.synchronize()
    with torch.cuda.graph(g1):
        held = vda.cross_attention(**x, lse=True)
    for _ in range(2):
        g1.replay()
        beside = other.cross_attention(**x, lse=True, stream=side)
    torch.cuda.synchronize()
    assert all(a.equal(b) and c.equal(b) for a, b, c in zip(held, want, beside))


def test_workspace_of_long_encoders():
    """Asked for where sums may move and not elsewhere; a call without it is refused."""
    vda = binding.Vda(64, "bf16")
    prm = lambda B=1, heads=1, cu=0: binding._CROSS_PARAMS.pack(binding._CROSS_PARAMS.size, B, heads, 1, 1.0, 0, cu, 0, 0, 0, 0, 0, 0, 0)  # noqa: E731
    need = lambda n, keys, p: vda.lib.vdn_vda_cross_attention_workspace_bytes(vda.h, n, keys, p)  # noqa: E731
    assert need(ROWS, 32768, prm()) == 0
    assert 0 < need(ROWS, 32769, prm()) <= 148 * 256 * 64 * 4
    assert need(400, 32769, prm(B=100)) > 0
    t = torch.zeros(64, device=DEV)
    assert need(200, 32768, prm(B=100, cu=t.data_ptr())) == 0 and need(200, 40000, prm(B=100, cu=t.data_ptr())) > 0
    p = t.data_ptr()
    assert vda.lib.vdn_vda_cross_attention(vda.h, p, p, p, p + 128, ROWS, 32769, prm(), None, 0, None) == 3
