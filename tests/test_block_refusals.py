"""What quantize, scaled_matmul and cross_attention refuse, without a GPU: the binding's checks on host tensors, and the C entry points'
on a null handle."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2609_20744_b200 import binding, build

E4M3, BF16, F32 = torch.float8_e4m3fn, torch.bfloat16, torch.float32
M, N, K = 6, 130, 160


def product():
    z = lambda *s, t=F32: torch.zeros(*s, dtype=t)
    return dict(a=z(2, 3, K, t=E4M3), a_scale=z(2, 3, 2), w=z(N, K, t=E4M3), w_scale=z(2, 2), bias=z(N), add=z(2, 3, N, t=BF16),
                out=z(2, 3, N, t=BF16))


def check_product(x):
    return binding.validate_matmul_args(BF16, 0, x["a"], x["a_scale"], x["w"], x["w_scale"], x["bias"], x["add"], x["out"], on_cuda=False)


def test_matching_operands_pass():
    assert check_product(product()) == (M, N, K, (K, K, N, N))
    x = product()
    x["bias"] = x["add"] = x["out"] = None
    assert check_product(x) == (M, N, K, (K, K, 0, N))
    x["a"] = torch.zeros(2, 3, K + 16, dtype=E4M3)[..., :K]
    x["w"] = torch.zeros(N, 2 * K, dtype=E4M3)[:, K:]
    assert check_product(x)[3] == (K + 16, 2 * K, 0, N)
    x["a"], x["a_scale"] = torch.zeros(K, dtype=E4M3), torch.zeros(2)
    assert check_product(x)[0] == 1
    odd = dict(product(), a=torch.zeros(2, 3, 176, dtype=E4M3)[..., :161], w=torch.zeros(N, 176, dtype=E4M3)[:, :161])
    assert check_product(odd)[2:] == (161, (176, 176, N, N))


@pytest.mark.parametrize("name,bad", [
    ("a", lambda x: x["a"].float()),
    ("a", lambda x: x["a"][..., ::2]),
    ("a", lambda x: torch.zeros(2, 3, K + 8, dtype=E4M3)[..., :K]),                # rows not at multiples of 16 bytes
    ("a", lambda x: torch.zeros(3, 2, K, dtype=E4M3).transpose(0, 1)),             # rows not evenly spaced
    ("a", lambda x: None),
    ("w", lambda x: x["w"][:, :-1].contiguous()),
    ("w", lambda x: x["w"][0]),
    ("a_scale", lambda x: x["a_scale"][..., :1].contiguous()),
    ("a_scale", lambda x: x["a_scale"].double()),
    ("w_scale", lambda x: x["w_scale"][:1].contiguous()),
    ("w_scale", lambda x: x["w_scale"].T),
    ("bias", lambda x: x["bias"].bfloat16()),
    ("bias", lambda x: x["bias"][:-1]),
    ("add", lambda x: x["add"].float()),
    ("add", lambda x: x["add"][:1]),
    ("out", lambda x: x["out"].float()),
    ("out", lambda x: torch.zeros(2, 3, N, 2, dtype=BF16)[..., 0]),
])
def test_mismatched_operand_is_refused(name, bad):
    x = product()
    x[name] = bad(x)
    with pytest.raises(ValueError, match=name):
        check_product(x)


def attention(packed=False):
    z = lambda *s, t=BF16: torch.zeros(*s, dtype=t)
    lead = (9,) if packed else (2, 5)
    x = dict(q=z(2, 3, 4, 64), k=z(*lead, 2, 64), v=z(*lead, 2, 64), mask=z(*lead, t=torch.bool), out=z(2, 3, 4, 64), lse=z(2, 3, 4, t=F32),
             cu_seqlens=None, lengths=None)
    x["cu_seqlens" if packed else "lengths"] = z(3 if packed else 2, t=torch.int32)
    return x


def check_attention(x):
    return binding.validate_cross_args(BF16, 64, 0, x["q"], x["k"], x["v"], x["cu_seqlens"], x["lengths"], x["mask"], x["out"], x["lse"],
                                       on_cuda=False)


def test_matching_states_pass():
    assert check_attention(attention()) == (2, 3, 5, 4, 2, (256, 128, 128, 256))
    assert check_attention(attention(True)) == (2, 3, 9, 4, 2, (256, 128, 128, 256))
    x = attention()
    both = torch.zeros(2, 5, 4, 64, dtype=BF16)
    x["k"], x["v"], x["q"], x["out"], x["lse"] = both[:, :, :2], both[:, :, 2:], torch.zeros(2, 4, 7, 4, 64, dtype=BF16), None, None
    assert check_attention(x) == (2, 28, 5, 4, 2, (256, 256, 256, 256))
    x["mask"] = x["lengths"] = None
    assert check_attention(x)[0] == 2


@pytest.mark.parametrize("packed,name,bad", [
    (False, "q", lambda x: x["q"].float()),
    (False, "q", lambda x: x["q"][..., :32].contiguous()),
    (False, "q", lambda x: x["q"][0, 0]),
    (False, "k", lambda x: x["k"][:, :, 0]),
    (False, "k", lambda x: x["k"][:1]),
    (False, "k", lambda x: torch.zeros(2, 5, 3, 64, dtype=BF16)),                  # 3 key heads for 4 heads
    (False, "k", lambda x: torch.zeros(5, 2, 2, 64, dtype=BF16).transpose(0, 1)),  # tokens not evenly spaced
    (True, "k", lambda x: torch.zeros(1, 9, 2, 64, dtype=BF16)),
    (False, "v", lambda x: x["v"][:, :4].contiguous()),
    (False, "v", lambda x: None),
    (False, "mask", lambda x: x["mask"].to(torch.uint8)),
    (False, "mask", lambda x: x["mask"][:, :4].contiguous()),
    (True, "mask", lambda x: x["mask"][None]),
    (False, "lengths", lambda x: x["lengths"].long()),
    (False, "lengths", lambda x: x["lengths"][:1]),
    (True, "lengths", lambda x: torch.zeros(2, dtype=torch.int32)),
    (True, "cu_seqlens", lambda x: x["cu_seqlens"][:2]),
    (False, "out", lambda x: x["out"].float()),
    (False, "lse", lambda x: x["lse"].bfloat16()),
    (False, "lse", lambda x: x["lse"].transpose(1, 2)),
])
def test_mismatched_state_is_refused(packed, name, bad):
    x = attention(packed)
    x[name] = bad(x)
    with pytest.raises(ValueError, match=name):
        check_attention(x)


def test_null_handle():
    build.build()
    lib = binding.load_library()
    q, m, c = (t(ctypes.sizeof(t)) for t in (binding.VdnQuantizeParams, binding.VdnMatmulParams, binding.VdnCrossParams))
    assert lib.vdn_vda_quantize(None, None, None, None, 1, 1, ctypes.byref(q), None) == 1
    assert lib.vdn_vda_scaled_matmul(None, None, None, None, 1, 1, 1, ctypes.byref(m), None) == 1
    assert lib.vdn_vda_cross_attention(None, None, None, None, None, 1, 1, ctypes.byref(c), None, 0, None) == 1
    assert lib.vdn_vda_cross_attention_workspace_bytes(None, 1, 1, ctypes.byref(c)) == 0


STRUCTS = ((binding.VdnQuantizeParams, binding._QUANTIZE_PARAMS, "vdn_vda_quantize_params"),
           (binding.VdnMatmulParams, binding._MATMUL_PARAMS, "vdn_vda_matmul_params"),
           (binding.VdnCrossParams, binding._CROSS_PARAMS, "vdn_vda_cross_params"))


def test_structs_match_the_header(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "s.c"
    sizes = ", ".join(f"sizeof({name})" for _, _, name in STRUCTS)
    src.write_text(f'#include <stdio.h>\n#include "vdn_vda.h"\nint main(void){{printf("%zu %zu %zu", {sizes}); return 0;}}\n')
    subprocess.run(["gcc", "-std=c99", f"-I{root}/include", str(src), "-o", str(tmp_path / "s")], check=True)
    got = subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in got] == [ctypes.sizeof(c) for c, _, _ in STRUCTS] == [p.size for _, p, _ in STRUCTS]
    for cls, packed, _ in STRUCTS:
        values = [1.5 if t is ctypes.c_float else i + 1 for i, (_, t) in enumerate(cls._fields_)]
        x = cls.from_buffer_copy(packed.pack(*values))
        assert [getattr(x, n) for n, _ in cls._fields_] == values
