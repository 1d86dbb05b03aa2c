"""quantize, scaled_matmul and cross_attention where their tiles, groups and choices of kernel meet, beside the layer they stand around, and
two calls at once.  Bounds as in test_gpu_block_ops."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as blk
from paper_2609_20744_b200 import binding, inputs
from tests.test_gpu_block_ops import (DEV, SIMT, TYPES, _built, check_attention, check_product, check_quantize, handle, np64, operands,  # noqa: F401
                                      product_bound, rng, states)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("H,Hk", [(3, 1), (12, 1), (31, 1), (33, 1), (40, 1), (36, 3), (70, 2), (96, 1), (200, 1)])
def test_many_heads_on_one_key_head(handle, dtype, d, H, Hk):
    """Groups that do not divide a warp's rows, and groups larger than it."""
    for lq, n in ((1, 130), (3, 77), (9, 200)):
        x, rows = states(2, lq, H, Hk, d, dtype, [n, 5], masked=0.2, seed=H + lq, lk=n)
        check_attention(handle(dtype, d), x, rows, dtype)


@pytest.mark.parametrize("dtype,d,flags", [("bf16", 128, 0), ("bf16", 64, 0), ("f32", 128, 0), ("bf16", 64, SIMT)])
@pytest.mark.parametrize("lq", [1, 70, 300])
def test_key_counts_around_tiles(handle, dtype, d, flags, lq):
    """Packed encoders that end in every part of a tile, neighbours' keys (here: NaN beyond the last) in the same tile."""
    lens = [1, 31, 32, 33, 63, 64, 65, 95, 96, 97, 127, 128, 129, 160, 255, 256, 257, 0, 384, 385]
    x, rows = states(len(lens), lq, 2, 1, d, dtype, lens, packed=True, seed=lq)
    check_attention(handle(dtype, d, flags), x, rows, dtype)
    x["mask"] = torch.zeros(x["k"].shape[0], dtype=torch.bool, device=DEV)
    for at in rows:                                                            # one key left in each, at its end
        if at.stop > at.start:
            x["mask"][at.stop - 1] = True
    x["k"], x["v"] = (torch.where(x["mask"][:, None, None], x[i], float("nan")) for i in ("k", "v"))
    check_attention(handle(dtype, d, flags), x, rows, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(300, 200, 208), (1031, 333, 130), (520, 127, 640)])
def test_products_of_many_rows_at_any_address(handle, dtype, m, n, k):
    """Results and what is added to them: both where tile copies reach, one of them, neither; apart and in place; without add."""
    vda = handle(dtype)
    x = operands(m, n, k, dtype, seed=m)
    first = check_product(vda, x, dtype)
    for pad_out in (-n % 8, 5, 1):
        room = torch.full((m, n + pad_out), 7.0, device=DEV, dtype=TYPES[dtype])
        check_product(vda, dict(x, add=None), dtype, out=room[:, :n])
        for pad_add in (-n % 8 + 8, 3):
            add = torch.full((m, n + pad_add), 9.0, device=DEV, dtype=TYPES[dtype])
            add[:, :n] = x["add"]
            got = vda.scaled_matmul(x["a"], x["a_scale"], x["w"], x["w_scale"], bias=x["bias"], add=add[:, :n], out=room[:, :n])
            assert got.equal(first) and (room[:, n:] == 7).all() and (add[:, n:] == 9).all()
        room[:, :n] = x["add"]
        got = vda.scaled_matmul(x["a"], x["a_scale"], x["w"], x["w_scale"], bias=x["bias"], add=room[:, :n], out=room[:, :n])
        assert got.equal(first) and (room[:, n:] == 7).all()
    shifted = torch.full((m * n + 8,), 7.0, device=DEV, dtype=TYPES[dtype])          # dense, but not from a multiple of 16 bytes on
    got = vda.scaled_matmul(x["a"], x["a_scale"], x["w"], x["w_scale"], bias=x["bias"], add=x["add"], out=shifted[1: 1 + m * n].view(m, n))
    assert got.equal(first) and (shifted[:1] == 7).all() and (shifted[1 + m * n:] == 7).all()


@pytest.mark.parametrize("m", [1, 40, 140, 300])
@pytest.mark.parametrize("k", [1, 17, 130, 255, 391])
def test_what_lies_between_rows_is_not_read(handle, m, k):
    """NaN in the bytes behind the channels of every row."""
    x = operands(m, 150, k, "bf16", seed=k)
    for name in ("a", "w"):
        room = torch.full((x[name].shape[0], -(-k // 16) * 16 + 16), float("nan"), device=DEV).to(x[name].dtype)
        room[:, :k] = x[name]
        x[name] = room[:, :k]
    check_product(handle("bf16"), x, "bf16")
    check_product(handle("bf16", flags=SIMT), x, "bf16")


def test_more_items_than_run_at_once(handle):
    """Persistent CTAs: batch rows of very uneven lengths one after another, some of them empty, odd numbers of tiles."""
    r = np.random.default_rng(0)
    for d, lq, H in ((128, 150, 4), (64, 400, 2)):
        lens = [int(n) if n > 20 else 0 for n in r.integers(0, 500, 180)]
        x, rows = states(len(lens), lq, H, H, d, "bf16", lens, packed=True, seed=d)
        check_attention(handle("bf16", d), x, rows, "bf16")


def test_parts_of_long_encoders(handle):
    """Few queries against long encoders, some batch rows too short for all of the parts."""
    for dtype, d, lq, H, Hk in (("bf16", 128, 5, 4, 2), ("bf16", 64, 130, 2, 1), ("f32", 64, 20, 2, 2), ("bf16", 128, 1, 3, 3)):
        lens = [4100, 0, 130, 2500]
        x, rows = states(4, lq, H, Hk, d, dtype, lens, masked=0.1, seed=lq)
        vda = handle(dtype, d)
        check_attention(vda, x, rows, dtype)
        assert vda.launch_count() == 2


def test_kernels_go_by_sizes(handle):
    vda = binding.Vda(128, "bf16")

    def kernel(f):
        vda.profile(True)
        f()
        torch.cuda.synchronize()
        name = vda.kernel_times()[0][0]
        vda.profile(False)
        return name

    def product(m, n=256, k=256):
        x = operands(m, n, k, "bf16")
        return kernel(lambda: vda.scaled_matmul(**x))

    def attention(lq, H, Hk, scale=None):
        x, _ = states(1, lq, H, Hk, 128, "bf16", [100])
        return kernel(lambda: vda.cross_attention(**x, scale=scale))

    assert [product(m) for m in (1, 64, 300, 2000)] == ["matmul_slim"] * 2 + ["matmul_pair"] * 2
    assert product(300, 130, 5000) == "matmul_slim" and product(1025, 130, 5000) == "matmul_pair"
    assert attention(1, 2, 2) == attention(2, 2, 2) == attention(1, 4, 2) == "cross_few"
    assert attention(3, 2, 2) == attention(1, 3, 1) == attention(500, 2, 2) == "cross_tc"
    assert attention(50, 2, 2, scale=-1.0) == "cross_plain" and attention(50, 2, 2, scale=1.0) == "cross_tc"


def test_two_calls_at_once():
    """Two handles, two streams, the large kernels of both in flight: as one after the other."""
    m = 3000
    x = operands(m, 1024, 512, "bf16", seed=1)
    y, _ = states(2, m, 4, 2, 128, "bf16", [300, 200], seed=2)
    act = torch.randn(m, 1024, generator=rng(3)).bfloat16().to(DEV)
    pair = [binding.Vda(128, "bf16") for _ in range(2)]

    def calls(vda, **kw):
        x8, s = vda.quantize(act, **kw)
        return [x8.view(torch.uint8), s, vda.scaled_matmul(**x, **kw), *vda.cross_attention(**y, lse=True, **kw)]

    want = calls(pair[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            got[i].append(calls(pair[i], stream=streams[i]))
    torch.cuda.synchronize()
    assert all(a.equal(b) for i in range(2) for c in got[i] for a, b in zip(c, want))
    assert all(v.status() == binding.VDN_OK for v in pair)


def test_a_new_call_while_a_captured_one_replays():
    vda = binding.Vda(128, "bf16")
    x, _ = states(1, 40, 2, 2, 128, "bf16", [3000], seed=4)                    # in parts: with a workspace
    want = [t.clone() for t in vda.cross_attention(**x, lse=True)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = vda.cross_attention(**x, lse=True)
    other, _ = states(1, 40, 2, 2, 128, "bf16", [3000], seed=5)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        g.replay()
        with torch.cuda.stream(side):
            fresh = vda.cross_attention(**other, lse=True)
    torch.cuda.synchronize()
    assert all(a.equal(b) for a, b in zip(held, want))
    assert all(a.equal(b) for a, b in zip(fresh, vda.cross_attention(**other, lse=True)))


def test_around_the_layer():
    """Tokens to q, k, v by one 8-bit projection, the layer's preparation and forward pass on them, its output projection, and the
    attention to a prompt projected and added to it (Eq. 1d's sum); every projection and the attention checked for its own inputs."""
    T, Y, X, H, d = 3, 4, 6, 2, 128
    n, wide = T * Y * X, H * d
    vda, w = binding.Vda(d, "bf16"), inputs.CLIP_480P.scaled(H=H, T=T, F=Y * X)
    g = rng(6)
    tokens = torch.randn(n, wide, generator=g).bfloat16().to(DEV)
    text = torch.randn(40, wide, generator=g).bfloat16().to(DEV)
    weight = lambda rows: vda.quantize((torch.randn(rows, wide, generator=g) * wide ** -0.5).bfloat16().to(DEV), rows=128)  # noqa: E731

    def project(x, wq, add=None):
        x8, s = check_quantize(vda, x, 1)
        y = vda.scaled_matmul(x8, s, *wq, add=add)
        want, size = blk.scaled_matmul(np64(x8), np64(s), np64(wq[0]), np64(wq[1]), add=np64(add))
        assert (np.abs(np64(y) - want) <= product_bound(want, size, "bf16", x.shape[1])).all()
        return y

    qkv = project(tokens, weight(3 * wide)).view(1, T, Y * X, 3 * H, d)
    q, k, v = (qkv[:, :, :, i * H: (i + 1) * H].contiguous() for i in range(3))
    extra = inputs.generate(w, DEV)
    filters = inputs.generate_projected(w, DEV)
    pq, pk, pv = vda.prepare(q, k, v, filters, Y, X)
    linear = vda.forward(pq, pk, pv, extra["beta"], extra["gate"])
    kv = project(text, weight(2 * wide)).view(1, 40, 2 * H, d)
    x = dict(q=q.view(1, n, H, d), k=kv[:, :, :H], v=kv[:, :, H:], mask=None, cu_seqlens=None, lengths=None)
    cross, _ = check_attention(vda, x, [(0, slice(0, 40))], "bf16")
    first = project(linear.view(n, wide), weight(wide))
    both = project(cross.view(n, wide), weight(wide), add=first)
    assert both.isfinite().all() and not both.equal(first)
    torch.cuda.synchronize()
    assert vda.status() == binding.VDN_OK


def test_refusals_of_sizes(handle):
    vda = handle("bf16")
    t = torch.zeros(4096, device=DEV)
    p = t.data_ptr()
    for scale in (float("inf"), -1e31, 2e30):
        prm = binding._CROSS_PARAMS.pack(binding._CROSS_PARAMS.size, 1, 1, 1, scale, 0, 0, 0, 0, 0, 0, 0, 0, 0)
        assert vda.lib.vdn_vda_cross_attention(vda.h, p, p + 4096, p + 4096, p + 8192, 1, 1, prm, 0, 0, None) == 1
        assert vda.lib.vdn_vda_cross_attention_workspace_bytes(vda.h, 1, 1, prm) == 0
    prm = binding._MATMUL_PARAMS.pack(binding._MATMUL_PARAMS.size, 0, p, p, 0, 0, 0, 0, 0, 0)
    for n, k in (((1 << 21) + 1, 32), (32, (1 << 21) + 16)):
        assert vda.lib.vdn_vda_scaled_matmul(vda.h, p, p + 4096, p + 8192, 1, n, k, prm, None) == 1
    with pytest.raises(ValueError, match="CUDA"):
        vda.quantize(torch.zeros(4, 32, dtype=torch.bfloat16))
