"""quantize, scaled_matmul and cross_attention against their 64-bit statements.

Tolerances.  u = 2^-8 (bf16) or 2^-24 (f32), half a step of the result; u32 = 2^-24.
  quantize: none, the codes and scales are equal.
  scaled_matmul, element by element: one rounding to io_dtype, u |out|; products of 8-bit numbers are exact, and a term passes
     through at most 128 additions in its block, one for each block, the scales' two roundings, bias and add, each off by u32, or by
     2 u32 where an addition cuts off: (128 + blocks + 5) 2 u32 times the sum of the terms' magnitudes.
  cross_attention: a score's d products and additions are off by at most dz = (2 d + 12) u32 times the sum of their magnitudes
     (`spread`, the largest of a row); that, the exponential (2^-21 with its argument's last rounding) and n additions of each sum
     give lse: dz + 2^-21 + 2 n u32 + 4 u32 |lse|.  out: u |out|, and relative to sum_j p_j |v_j| (`weight`) twice the above, and u16
     = 2^-8 where weights are rounded to bf16 for the tensor cores.
"""
import numpy as np
import pytest
import torch

from oracle import block_oracle as blk
from paper_2609_20744_b200 import binding, build

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
U16, U32 = 2.0 ** -8, 2.0 ** -24
E4M3 = torch.float8_e4m3fn
SIMT = binding.VDN_FLAG_FORCE_SIMT


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.load_library()


@pytest.fixture(scope="module")
def handle():
    made = {}

    def get(dtype="bf16", d=128, flags=0):
        if (dtype, d, flags) not in made:
            made[dtype, d, flags] = binding.Vda(d, dtype, flags=flags)
        return made[dtype, d, flags]

    yield get
    torch.cuda.synchronize()
    assert all(v.status() == binding.VDN_OK for v in made.values())


def np64(x):
    return None if x is None else x.detach().double().cpu().numpy()


def rng(seed):
    return torch.Generator().manual_seed(seed)


# ------------------------------------------------------------------------------------------------ quantize
def check_quantize(vda, x, rows, **kw):
    x8, s = vda.quantize(x, rows=rows, **kw)
    want, ws = blk.quantize(np64(x).reshape(-1, x.shape[-1]), rows)
    assert x8.dtype is E4M3 and x8.shape == x.shape and s.dtype is torch.float32
    assert np.array_equal(np64(s).reshape(ws.shape), ws)
    got = np64(x8).reshape(want.shape)
    assert np.array_equal(got, want, equal_nan=True)
    assert np.array_equal(np.signbit(got), np.signbit(want)) or np.isnan(want).any()
    return x8, s


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("shape", [(1, 1), (1, 128), (3, 7), (5, 129), (128, 128), (129, 255), (33, 1000), (200, 641), (700, 136)])
def test_quantize(handle, dtype, rows, shape):
    x = torch.randn(shape, generator=rng(1)) * torch.exp(4 * torch.randn(shape[0], 1, generator=rng(2)))
    check_quantize(handle(dtype), x.to(TYPES[dtype]).to(DEV), rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_at_the_edges_of_the_range(handle, dtype, rows):
    """Blocks of zeros, of the smallest and largest numbers, maxima on both sides of a power of two times 448, ties, and what is not
    finite."""
    big = torch.finfo(TYPES[dtype]).max
    x = torch.randn(12, 260, generator=rng(3))
    x[0] = 0
    x[1] = -0.0
    x[2] = x[2].sign() * 2.0 ** -133
    x[3] *= 2.0 ** -125
    x[4] = big
    x[5, ::2] = -big
    x[6] = torch.arange(260) / 16 + 448 - 4
    x[7, 0], x[7, 128], x[7, 256] = 448.0, 450.0, 446.0
    x[8, :7] = torch.tensor([448.0, 17.0, 19.0, 21.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -11])
    x[9, 3], x[9, 130], x[9, 259] = float("inf"), -float("inf"), float("nan")
    x[10] = float("inf")
    x[11] = float("nan")
    x = x.to(TYPES[dtype]).to(DEV)
    for part in (x, x[:9].contiguous(), x[9:].contiguous(), *(x[i: i + 1] for i in range(12))):
        check_quantize(handle(dtype), part, rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_of_slices_into_given_memory(handle, dtype):
    vda, dt = handle(dtype), TYPES[dtype]
    wide = torch.randn(6, 5, 400, generator=rng(4)).to(dt).to(DEV)
    check_quantize(vda, wide[..., 8:208], 1)
    check_quantize(vda, wide[..., 3:160], 1)                                     # rows that begin anywhere
    check_quantize(vda, wide[:, 0, 1:301], 128)
    check_quantize(vda, wide[0, 0], 1)                                           # a single row without a leading dimension
    room = torch.full((40, 176), 3.0, device=DEV).to(E4M3)
    scale = torch.full((40, 2), 5.0, device=DEV)
    x = torch.randn(37, 150, generator=rng(5)).to(dt).to(DEV)
    check_quantize(vda, x, 1, out=room[:37, :150], scale=scale[:37])
    assert (room[37:].float() == 3).all() and (room[:, 150:].float() == 3).all() and (scale[37:] == 5).all()
    x8, s = vda.quantize(x[:0])
    assert x8.shape == (0, 150) and s.shape == (0, 2)


# ------------------------------------------------------------------------------------------------ scaled_matmul
def operands(m, n, k, dtype, seed=0, bias=True, add=True, lead=None, pow2=False):
    g = rng(seed)
    rows = -(-k // 16) * 16
    e = lambda r: (torch.randn(r, rows, generator=g) * torch.exp2(4 * torch.randn(r, 1, generator=g))).clamp(-448, 448).to(E4M3)
    s = lambda *shape: torch.exp2(torch.randn(shape, generator=g).round()) if pow2 else torch.exp(torch.randn(shape, generator=g))
    blocks = -(-k // 128)
    x = dict(a=e(m), a_scale=s(m, blocks), w=e(n), w_scale=s(-(-n // 128), blocks) / k)
    x["bias"] = torch.randn(n, generator=g) if bias else None
    x["add"] = torch.randn(m, n, generator=g).to(TYPES[dtype]) if add else None
    x = {i: None if t is None else t.to(DEV) for i, t in x.items()}
    x["a"], x["w"] = x["a"][:, :k], x["w"][:, :k]
    return x


def product_bound(want, size, dtype, k):
    return U[dtype] * np.abs(want) + (128 + -(-k // 128) + 5) * 2 * U32 * size


def check_product(vda, x, dtype, **kw):
    want, size = blk.scaled_matmul(*(np64(x[i]) for i in ("a", "a_scale", "w", "w_scale", "bias", "add")))
    got = vda.scaled_matmul(x["a"], x["a_scale"], x["w"], x["w_scale"], bias=x["bias"], add=x["add"], **kw)
    assert got.dtype is TYPES[dtype]
    assert (np.abs(np64(got) - want) <= product_bound(want, size, dtype, x["a"].shape[1])).all()
    return got


PRODUCTS = [(1, 1, 1), (1, 128, 128), (2, 64, 16), (3, 7, 130), (7, 513, 300), (16, 128, 512), (17, 129, 129), (33, 640, 1160), (64, 256, 384),
            (65, 1001, 77), (128, 128, 128), (129, 384, 2048), (130, 130, 1352), (200, 72, 4000), (257, 511, 257), (300, 1024, 1024)]


@pytest.mark.parametrize("dtype,flags", [("bf16", 0), ("f32", 0), ("bf16", SIMT), ("f32", SIMT)])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(handle, dtype, flags, m, n, k):
    vda = handle(dtype, flags=flags)
    check_product(vda, operands(m, n, k, dtype, seed=m + n + k), dtype)
    check_product(vda, operands(m, n, k, dtype, seed=m, bias=False, add=False, pow2=True), dtype)


@pytest.mark.parametrize("m", [1, 5, 8, 9, 24, 40, 63, 96, 127])
def test_product_of_few_rows_and_a_long_sum(handle, m):
    check_product(handle("f32"), operands(m, 320, 9000, "f32", seed=m), "f32")


@pytest.mark.parametrize("m,n,k", [(1500, 1100, 640), (4099, 260, 200), (140, 9000, 136), (20000, 129, 128)])
def test_product_of_many_tiles(handle, m, n, k):
    """More tiles than the GPU runs at once."""
    check_product(handle("bf16"), operands(m, n, k, "bf16", seed=k), "bf16")


@pytest.mark.parametrize("dtype,flags", [("bf16", 0), ("f32", 0), ("bf16", SIMT)])
@pytest.mark.parametrize("m", [3, 140])
def test_product_of_slices_in_place(handle, dtype, flags, m):
    vda, n, k = handle(dtype, flags=flags), 200, 208
    x = operands(m, n, k, dtype, seed=9)
    wide = lambda t, pad: torch.cat((t.float(), torch.full((t.shape[0], pad), 99.0, device=DEV)), 1).to(t.dtype)
    x["a"], x["w"] = wide(x["a"], 32)[:, :k], wide(x["w"], 16)[:, :k]
    plain = check_product(vda, x, dtype)
    for pad in (8, 5, 1):                                                      # rows of the results that begin anywhere
        room = torch.full((m, n + pad), 7.0, device=DEV, dtype=TYPES[dtype])
        room[:, :n] = x["add"]
        assert check_product(vda, dict(x, add=room[:, :n]), dtype, out=torch.empty_like(room)[:, :n]).equal(plain)
        got = vda.scaled_matmul(x["a"], x["a_scale"], x["w"], x["w_scale"], bias=x["bias"], add=room[:, :n], out=room[:, :n])
        assert got.data_ptr() == room.data_ptr() and got.equal(plain) and (room[:, n:] == 7).all()
    lead = vda.scaled_matmul(x["a"][None], x["a_scale"][None], x["w"], x["w_scale"], bias=x["bias"], add=x["add"][None])
    assert lead.shape == (1, m, n) and lead[0].equal(plain)
    assert vda.scaled_matmul(x["a"][:0], x["a_scale"][:0], x["w"], x["w_scale"]).shape == (0, n)


@pytest.mark.parametrize("m", [4, 150])
def test_product_leaves_a_row_that_is_not_finite_to_itself(handle, m):
    vda = handle("bf16")
    x = operands(m, 300, 400, "bf16", seed=11)
    clean = check_product(vda, x, "bf16")
    a = x["a"].float()
    a[1, 399] = float("nan")
    w = x["w"].float()
    w[7, 0] = float("nan")
    s = x["a_scale"].clone()
    s[2, 1] = float("inf")
    pitch = torch.zeros(m, 400, device=DEV).to(E4M3)
    pitch[:] = a.to(E4M3)
    got = vda.scaled_matmul(pitch, s, w.to(E4M3), x["w_scale"], bias=x["bias"], add=x["add"])
    rows = [i for i in range(m) if i not in (1, 2)]
    cols = [i for i in range(300) if i != 7]
    assert got[rows][:, cols].equal(clean[rows][:, cols])
    assert got[1].isnan().all() and got[:, 7].isnan().all() and not got[2].isfinite().any()


@pytest.mark.parametrize("m", [2, 60, 700])
def test_product_same_call_same_bits(handle, m):
    vda, x = handle("f32"), operands(m, 1000, 1500, "f32", seed=13)
    first = vda.scaled_matmul(**x)
    for _ in range(20):
        assert vda.scaled_matmul(**x).equal(first)


# ------------------------------------------------------------------------------------------------ cross_attention
def states(B, lq, H, Hk, d, dtype, lens, packed=False, masked=0.0, seed=0, lk=None):
    """q, k, v and how the keys of each batch row are told; what does not count is NaN."""
    g = rng(seed)
    rand = lambda *s: torch.randn(*s, generator=g)
    lk = max(lens, default=0) if lk is None else lk
    lead = (sum(lens) + 3,) if packed else (B, lk)
    x = dict(q=rand(B, lq, H, d), k=1.5 * rand(*lead, Hk, d), v=rand(*lead, Hk, d))
    counts = torch.zeros(lead, dtype=torch.bool)
    cu = torch.tensor([0] + list(lens)).cumsum(0)
    for b, n in enumerate(lens):
        if packed:
            counts[cu[b]: cu[b + 1]] = True
        else:
            counts[b, :n] = True
    mask = None
    if masked:
        mask = torch.rand(lead, generator=g) >= masked
        counts &= mask
    x["k"][~counts] = float("nan")
    x["v"][~counts] = float("nan")
    x = {n: t.to(TYPES[dtype]).to(DEV) for n, t in x.items()}
    x["mask"] = None if mask is None else mask.to(DEV)
    x["cu_seqlens"] = cu.to(torch.int32).to(DEV) if packed else None
    x["lengths"] = None if packed or (not masked and all(n == lk for n in lens)) else torch.tensor(lens, dtype=torch.int32).to(DEV)
    rows = [(slice(int(cu[b]), int(cu[b + 1])) if packed else (b, slice(0, n))) for b, n in enumerate(lens)]
    return x, rows



def check_attention(vda, x, rows, dtype, scale=None, **kw):
    out, lse = vda.cross_attention(**x, scale=scale, lse=True, **kw)
    assert out.shape == x["q"].shape and out.dtype is TYPES[dtype] and lse.shape == x["q"].shape[:-1]
    B, d = x["q"].shape[0], x["q"].shape[-1]
    q, got, glse = np64(x["q"]).reshape(B, -1, *x["q"].shape[-2:]), np64(out), np64(lse)
    got, glse = got.reshape(q.shape), glse.reshape(q.shape[:-1])
    for b, at in enumerate(rows):
        counts = None if x["mask"] is None else x["mask"][at].cpu().numpy()
        k, v = np64(x["k"][at]), np64(x["v"][at])
        want, wlse, spread, weight = blk.cross_attention(q[b], k, v, d ** -0.5 if scale is None else scale, counts)
        n = k.shape[0]
        dz = (2 * d + 12) * U32 * spread + 2.0 ** -21 + 2 * n * U32
        bound = U[dtype] * np.abs(want) + weight * (2 * dz[..., None] + (U16 if dtype == "bf16" else 0))
        assert (np.abs(got[b] - want) <= bound).all()
        some = np.isfinite(wlse)
        assert np.array_equal(glse[b][~some], wlse[~some])
        assert (np.abs(glse[b][some] - wlse[some]) <= dz[some] + 4 * U32 * np.abs(wlse[some])).all()
    return out, lse


KINDS = [("bf16", 128, 0), ("bf16", 64, 0), ("f32", 128, 0), ("f32", 64, 0), ("bf16", 128, SIMT), ("bf16", 64, SIMT)]
SHAPES = [  # batch, queries, heads, key heads, keys of each row
    (1, 1, 1, 1, [1]), (1, 1, 4, 4, [77]), (2, 1, 6, 2, [129, 64]), (3, 1, 8, 1, [300, 0, 1]), (1, 3, 8, 4, [1000]),
    (1, 8, 2, 2, [500]), (1, 9, 2, 1, [130]), (1, 64, 3, 3, [128]), (2, 127, 2, 1, [77, 128]), (1, 128, 1, 1, [256]), (1, 129, 2, 2, [257]),
    (3, 300, 4, 2, [40, 0, 513]), (1, 257, 6, 2, [200]), (2, 50, 12, 1, [3, 700]), (1, 1000, 2, 2, [64]), (1, 20, 2, 2, [3000])]


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("B,lq,H,Hk,lens", SHAPES)
def test_attention(handle, dtype, d, flags, B, lq, H, Hk, lens):
    vda = handle(dtype, d, flags)
    for packed, masked in ((False, 0.0), (True, 0.0), (False, 0.4)):
        x, rows = states(B, lq, H, Hk, d, dtype, lens, packed, masked, seed=lq + H)
        check_attention(vda, x, rows, dtype)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("lq", [1, 5, 200])
def test_attention_rows_without_keys(handle, dtype, d, flags, lq):
    """No key counts: by the mask alone, by a length of zero, with no key tensor to speak of, in parts of a long row."""
    vda = handle(dtype, d, flags)
    x, rows = states(3, lq, 4, 2, d, dtype, [5, 0, 400], masked=0.3, lk=400)
    x["mask"][0] = False
    x["k"][0], x["v"][0] = float("nan"), float("inf")
    out, lse = check_attention(vda, x, rows, dtype)
    assert (out[:2] == 0).all() and (lse[:2] == -float("inf")).all() and lse[2].isfinite().all()
    x["mask"][2, 7:] = False                                                     # keys only in the first of several parts
    x["mask"][2, 3] = True
    x["k"][2, 3], x["v"][2, 3] = 1.0, 2.0
    x["k"][2, :7] = torch.where(x["k"][2, :7].isnan(), 0.5, x["k"][2, :7])
    x["v"][2, :7] = torch.where(x["v"][2, :7].isnan(), 0.5, x["v"][2, :7])
    check_attention(vda, x, rows, dtype)
    x, rows = states(2, lq, 4, 2, d, dtype, [0, 0], lk=0)
    out, lse = check_attention(vda, x, rows, dtype)
    assert (out == 0).all() and (lse == -float("inf")).all()
    x, rows = states(2, lq, 4, 2, d, dtype, [0, 0], packed=True)
    check_attention(vda, x, rows, dtype)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("lq", [2, 130])
def test_attention_scores_of_any_size(handle, dtype, d, flags, lq):
    """A maximum that grows from tile to tile, or sits in the first; scores of -1e4 throughout; equal scores; no scale; a negative one."""
    vda = handle(dtype, d, flags)
    n = 600
    x, rows = states(1, lq, 2, 2, d, dtype, [n], seed=3)
    grow = torch.linspace(0.02, 4, n, device=DEV)[None, :, None, None]
    for factor in (grow, grow.flip(1)):
        check_attention(vda, dict(x, k=(x["k"].float() * factor).to(TYPES[dtype])), rows, dtype)
    far = x["k"].clone()
    far[..., 0] = -100.0
    x["q"][..., 0] = 100.0 * d ** 0.5
    check_attention(vda, dict(x, k=far), rows, dtype)
    out, lse = check_attention(vda, dict(x, k=torch.ones_like(far)), rows, dtype)
    check_attention(vda, x, rows, dtype, scale=0.0)
    check_attention(vda, x, rows, dtype, scale=-0.3 * d ** -0.5)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("lq", [3, 140])
def test_attention_of_slices_into_given_memory(handle, dtype, d, flags, lq):
    vda, dt, n, H, Hk = handle(dtype, d, flags), TYPES[dtype], 210, 4, 2
    both = torch.randn(2, n, 2 * Hk, d, generator=rng(6)).to(dt).to(DEV)        # one projection's keys and values
    three = torch.randn(2, lq, 3 * H, d, generator=rng(7)).to(dt).to(DEV)
    x = dict(q=three[:, :, H: 2 * H], k=both[:, :, :Hk], v=both[:, :, Hk:], mask=None, cu_seqlens=None, lengths=None)
    rows = [(b, slice(0, n)) for b in range(2)]
    room = torch.full((2, lq, H + 1, d), 7.0, device=DEV, dtype=dt)
    out, lse = check_attention(vda, x, rows, dtype, out=room[:, :, :H])
    assert out.data_ptr() == room.data_ptr() and (room[:, :, H:] == 7).all()
    given = torch.full((2, lq, H), 3.0, device=DEV)
    again, same = vda.cross_attention(x["q"], x["k"], x["v"], lse=given)
    assert same is given and again.equal(out) and given.equal(lse)
    assert vda.cross_attention(x["q"], x["k"], x["v"]).equal(out)
    if lq == 140:                                                                # queries of a clip [B, T, F, H, d]
        clip = x["q"].contiguous().view(2, 7, 20, H, d)
        y, z = vda.cross_attention(clip, x["k"], x["v"], lse=True)
        assert y.shape == clip.shape and z.shape == clip.shape[:-1] and y.view(2, lq, H, d).equal(out)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("lq", [1, 150])
def test_attention_a_row_that_is_not_finite_stays_alone(handle, dtype, d, flags, lq):
    vda = handle(dtype, d, flags)
    x, rows = states(3, lq, 4, 2, d, dtype, [260, 260, 260], seed=8)
    out, lse = check_attention(vda, x, rows, dtype)
    q, k, v = (x[i].clone() for i in ("q", "k", "v"))
    q[0, 0, 1] = float("nan")
    k[1, 130, 0] = float("nan")                                                  # key head 0 of batch row 1: heads 0 and 1
    v[2, 5, 1, 3] = float("inf")                                                 # one channel of heads 2 and 3
    got, glse = vda.cross_attention(q, k, v, lse=True)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[0, 0, 1], bad[1, :, :2], bad[2, :, 2:, 3] = True, True, True
    assert not got[bad].isfinite().any() and got[~bad].equal(out[~bad])
    assert glse[2].equal(lse[2]) and glse[1, :, :2].isnan().all() and glse[0, 0, 1].isnan()


@pytest.mark.parametrize("dtype,d,flags", KINDS)
def test_attention_clamps_lengths_and_offsets(handle, dtype, d, flags):
    vda = handle(dtype, d, flags)
    for lq in (1, 140):
        x, rows = states(2, lq, 2, 2, d, dtype, [50, 50], seed=9)
        whole = vda.cross_attention(**x)
        got = vda.cross_attention(x["q"], x["k"], x["v"], lengths=torch.tensor([10 ** 9, -4], dtype=torch.int32, device=DEV))
        assert got[0].equal(whole[0]) and (got[1] == 0).all()
        k, v = x["k"].flatten(0, 1), x["v"].flatten(0, 1)
        got = vda.cross_attention(x["q"], k, v, cu_seqlens=torch.tensor([-5, 50, 10 ** 9], dtype=torch.int32, device=DEV))
        assert got.equal(whole)


@pytest.mark.parametrize("dtype,d,flags", KINDS)
@pytest.mark.parametrize("B,lq,n", [(1, 1, 5000), (2, 30, 2000), (1, 700, 400)])
def test_attention_same_call_same_bits(handle, dtype, d, flags, B, lq, n):
    vda = handle(dtype, d, flags)
    x, _ = states(B, lq, 4, 2, d, dtype, [n] * B, seed=10)
    first = vda.cross_attention(**x, lse=True)
    for _ in range(20):
        again = vda.cross_attention(**x, lse=True)
        assert again[0].equal(first[0]) and again[1].equal(first[1])


# ------------------------------------------------------------------------------------------------ streams, graphs, long tensors
def a_call_of_each(vda, dtype, d, m):
    x = operands(m, 160, 256, dtype, seed=m)
    y, _ = states(2, m, 4, 2, d, dtype, [300, 77], seed=m, lk=300)
    act = torch.randn(m, 256, generator=rng(m)).to(TYPES[dtype]).to(DEV)

    def call(**kw):
        x8, s = vda.quantize(act, **kw)
        z = vda.scaled_matmul(x8, s, x["w"], x["w_scale"], bias=x["bias"], add=x["add"], **kw)
        return (x8.view(torch.uint8), s, z, *vda.cross_attention(**y, lse=True, **kw))

    return call, act, x, y


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("m", [1, 140])
def test_calls_on_another_stream(dtype, d, m):
    vda = binding.Vda(d, dtype)
    call, act, _, _ = a_call_of_each(vda, dtype, d, m)
    want = [t.clone() for t in call()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        later = act.clone()
        act.zero_()
        act.copy_(later)
    got = call(stream=side)                                                      # ordered behind the copy by the stream alone
    junk = [torch.full((1 << 20,), 9.0, device=DEV) for _ in range(4)]            # what the allocator hands out meanwhile
    torch.cuda.current_stream().wait_stream(side)
    assert all(a.equal(b) for a, b in zip(got, want))
    del junk
    torch.cuda.synchronize()
    assert vda.status() == binding.VDN_OK


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("m", [1, 140])
def test_calls_captured_twice_and_replayed_on_new_inputs(dtype, d, m):
    vda = binding.Vda(d, dtype)
    call, act, x, y = a_call_of_each(vda, dtype, d, m)
    call()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call())
        graphs.append(g)
    act.mul_(0.5)
    y["v"].mul_(3)
    y["lengths"].copy_(torch.tensor([10, 200], dtype=torch.int32))
    y["v"].nan_to_num_()
    y["k"].nan_to_num_()
    want = [t.clone() for t in call()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):                                                           # both at once
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
    torch.cuda.synchronize()
    assert all(a.equal(b) for o in outs for a, b in zip(o, want))
    assert vda.status() == binding.VDN_OK


def test_offsets_beyond_32_bits(handle):
    """Tensors of more than 2^31 elements: the last rows against the same rows in a small tensor."""
    vda, m, k = handle("bf16"), 270_000, 8192
    x = torch.zeros(m, k, device=DEV, dtype=torch.bfloat16)
    x[-300:] = torch.randn(300, k, generator=rng(1)).bfloat16().to(DEV)
    w, ws = vda.quantize(torch.randn(136, k, generator=rng(2)).bfloat16().to(DEV), rows=128)
    x8, s = vda.quantize(x)
    tail8, tail_s = vda.quantize(x[-300:].clone())
    assert x8[-300:].view(torch.uint8).equal(tail8.view(torch.uint8)) and s[-300:].equal(tail_s)
    got = vda.scaled_matmul(x8, s, w, ws)
    want, size = blk.scaled_matmul(np64(tail8), np64(tail_s), np64(w), np64(ws))
    assert (np.abs(np64(got[-300:]) - want) <= product_bound(want, size, "bf16", k)).all() and (got[:-300] == 0).all()
    del x8, got
    q = x.view(1, m, 64, 128)                                                    # the same memory as queries, then as keys
    state = torch.randn(1, 70, 64, 128, generator=rng(3)).bfloat16().to(DEV)
    out = vda.cross_attention(q, state, state)
    assert out[:, -300:].equal(vda.cross_attention(q[:, -300:].contiguous(), state, state))
    del out
    cu = torch.tensor([0, m - 300, m], dtype=torch.int32, device=DEV)
    few = torch.randn(2, 2, 64, 128, generator=rng(4)).bfloat16().to(DEV)
    many = few.repeat(1, 70, 1, 1)
    for queries in (few, many):
        got = vda.cross_attention(queries, q[0], q[0], cu_seqlens=cu)
        want = vda.cross_attention(queries[1:], q[:, -300:].contiguous(), q[:, -300:].contiguous())
        assert (got[1:].float() - want.float()).abs().max() <= 4 * U16 * x[-300:].float().abs().max()   # (cut in other parts)
        assert (got[0] == 0).all()
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("tokens", [1, 150])
def test_a_block_from_tokens_to_the_residual(handle, dtype, d, tokens):
    """Queries of the tokens and keys and values of a prompt by 8-bit projections, attention, and the output projection added to the
    tokens; each step's result checked for the very inputs it had."""
    vda, B, H, prompt, wide = handle(dtype, d), 2, 4, 90, 4 * d
    g = rng(20)
    act = torch.randn(B, tokens, wide, generator=g).to(TYPES[dtype]).to(DEV)
    text = torch.randn(B, prompt, 200, generator=g).to(TYPES[dtype]).to(DEV)
    weights = [vda.quantize((torch.randn(n, k, generator=g) * k ** -0.5).to(TYPES[dtype]).to(DEV), rows=128)
               for n, k in ((wide, wide), (2 * wide, 200), (wide, wide))]

    def project(x, w, add=None, out=None):
        x8, s = check_quantize(vda, x, 1)
        flat = lambda t: None if t is None else t.reshape(-1, t.shape[-1])
        y = vda.scaled_matmul(x8, s, *w, add=add, out=out)
        want, size = blk.scaled_matmul(np64(flat(x8)), np64(flat(s)), np64(w[0]), np64(w[1]), add=np64(flat(kept)) if add is not None else None)
        assert (np.abs(np64(flat(y)) - want) <= product_bound(want, size, dtype, x.shape[-1])).all()
        return y

    q = project(act, weights[0]).view(B, tokens, H, d)
    kv = project(text, weights[1]).view(B, prompt, 2 * H, d)
    x = dict(q=q, k=kv[:, :, :H], v=kv[:, :, H:], mask=None, cu_seqlens=None, lengths=torch.tensor([prompt, 33], dtype=torch.int32, device=DEV))
    out, _ = check_attention(vda, x, [(0, slice(0, prompt)), (1, slice(0, 33))], dtype)
    kept = act.clone()
    y = project(out.view(B, tokens, wide), weights[2], add=act, out=act)
    assert y.data_ptr() == act.data_ptr() and not y.equal(kept)


def test_refusals_with_a_handle(handle):
    vda = handle("bf16")
    lib, h = vda.lib, vda.h
    t = torch.zeros(4096, device=DEV)
    p = t.data_ptr()

    def refused(status, f, *args):
        before = t.clone()
        assert f(h, *args) == status
        assert vda.lib.vdn_vda_last_error(h)
        torch.cuda.synchronize()
        assert t.equal(before)

    def quantize(size=binding._QUANTIZE_PARAMS.size, rows=1, xs=0, os=0):
        return binding._QUANTIZE_PARAMS.pack(size, rows, xs, os)

    f = lib.vdn_vda_quantize
    for status, args in ((1, (p, p + 4096, p + 8192, 4, 32, None, None)), (1, (p, p + 4096, p + 8192, 4, 32, quantize(8), None)),
                         (1, (p, p + 4096, p + 8192, 4, 32, quantize(rows=2), None)), (1, (p, p + 4096, p + 8192, 4, 0, quantize(), None)),
                         (1, (p, p + 4096, p + 8192, -1, 32, quantize(), None)), (1, (0, p + 4096, p + 8192, 4, 32, quantize(), None)),
                         (1, (p, p + 4100, p + 8192, 4, 32, quantize(), None)), (1, (p + 1, p + 4096, p + 8192, 4, 32, quantize(), None)),
                         (1, (p, p + 4096, p + 8192, 4, 40, quantize(), None)), (1, (p, p, p + 8192, 4, 32, quantize(), None)),
                         (1, (p, p + 4096, p + 8192, 4, 32, quantize(xs=16), None)), (1, (p, p + 4096, p + 8192, 4, 32, quantize(os=40), None)),
                         (2, (p, p + 4096, p + 8192, 1 << 30, 1024, quantize(), None))):
        refused(status, f, *args)

    def matmul(size=binding._MATMUL_PARAMS.size, reserved=0, sa=p, sw=p, bias=0, add=0, st=(0, 0, 0, 0)):
        return binding._MATMUL_PARAMS.pack(size, reserved, sa, sw, bias, add, *st)

    f = lib.vdn_vda_scaled_matmul
    a, w, o = p + 1024, p + 2048, p + 4096
    for args in ((a, w, o, 4, 4, 32, None, None), (a, w, o, 4, 4, 32, matmul(4), None), (a, w, o, 4, 4, 32, matmul(reserved=1), None),
                 (a, w, o, -1, 4, 32, matmul(), None), (a, w, o, 4, 0, 32, matmul(), None), (a, w, o, 4, 4, 0, matmul(), None),
                 (a, w, o, 4, 4, 1 << 23, matmul(), None), (0, w, o, 4, 4, 32, matmul(), None), (a, w, o, 4, 4, 32, matmul(sa=0), None),
                 (a + 8, w, o, 4, 4, 32, matmul(), None), (a, w + 1, o, 4, 4, 32, matmul(), None), (a, w, o + 1, 4, 4, 32, matmul(), None),
                 (a, w, a, 4, 4, 32, matmul(), None), (a, w, o, 4, 4, 40, matmul(), None), (a, w, o, 4, 4, 32, matmul(st=(16, 0, 0, 0)), None),
                 (a, w, o, 4, 4, 32, matmul(st=(0, 40, 0, 0)), None), (a, w, o, 4, 4, 32, matmul(st=(0, 0, 0, 3)), None),
                 (a, w, o, 4, 4, 32, matmul(add=o, st=(0, 0, 8, 4)), None), (a, w, o, 4, 4, 32, matmul(bias=p + 2), None)):
        refused(1, f, *args)

    def cross(size=binding._CROSS_PARAMS.size, B=1, H=2, Hk=1, scale=1.0, reserved=0, cu=0, lens=0, mask=0, lse=0, st=(0, 0, 0, 0)):
        return binding._CROSS_PARAMS.pack(size, B, H, Hk, scale, reserved, cu, lens, mask, lse, *st)

    f = lib.vdn_vda_cross_attention
    q, k, o = p, p + 4096, p + 8192
    for status, args in ((1, (q, k, k, o, 1, 1, None, 0, 0, None)), (1, (q, k, k, o, 1, 1, cross(8), 0, 0, None)),
                         (1, (q, k, k, o, 1, 1, cross(Hk=0), 0, 0, None)), (1, (q, k, k, o, 1, 1, cross(H=3, Hk=2), 0, 0, None)),
                         (1, (q, k, k, o, 1, 1, cross(scale=float("nan")), 0, 0, None)), (1, (q, k, k, o, 1, 1, cross(reserved=1), 0, 0, None)),
                         (1, (q, k, k, o, -1, 1, cross(), 0, 0, None)), (1, (q, k, k, o, 1, -1, cross(), 0, 0, None)),
                         (1, (q, k, k, o, 1, 1, cross(B=-1), 0, 0, None)), (1, (q, k, k, o, 1, 1, cross(cu=p, lens=p), 0, 0, None)),
                         (1, (0, k, k, o, 1, 1, cross(), 0, 0, None)), (1, (q, 0, k, o, 1, 1, cross(), 0, 0, None)),
                         (1, (q + 8, k, k, o, 1, 1, cross(), 0, 0, None)), (1, (q, k, k, q, 1, 1, cross(), 0, 0, None)),
                         (1, (q, k, k, k, 1, 1, cross(), 0, 0, None)), (1, (q, k, k, o, 1, 1, cross(st=(128, 0, 0, 0)), 0, 0, None)),
                         (1, (q, k, k, o, 1, 1, cross(st=(0, 132, 0, 0)), 0, 0, None)), (1, (q, k, k, o, 1, 1, cross(), p + 4, 64, None)),
                         (1, (q, k, k, o, 1 << 31, 1, cross(), 0, 0, None)), (2, (q, k, k, o, 1, 1, cross(H=70000), 0, 0, None)),
                         (3, (q, k, k, o, 1, 100000, cross(), 0, 0, None)), (3, (q, k, k, o, 1, 100000, cross(), p, 64, None))):
        refused(status, f, *args)
    assert vda.cross_attention(torch.zeros(0, 5, 2, 128, device=DEV, dtype=torch.bfloat16),
                               torch.zeros(0, 3, 1, 128, device=DEV, dtype=torch.bfloat16),
                               torch.zeros(0, 3, 1, 128, device=DEV, dtype=torch.bfloat16)).shape == (0, 5, 2, 128)
    with pytest.raises(ValueError):
        vda.quantize(torch.zeros(4, 32, device=DEV, dtype=torch.bfloat16), rows=2)
    with pytest.raises(ValueError):
        vda.quantize(torch.zeros(2, 4, 32, device=DEV, dtype=torch.bfloat16), rows=128)
