"""What token_scan, token_step and rotate refuse, without a GPU: the binding's checks on host tensors, and the C entry points'
on a null handle."""
import ctypes

import pytest
import torch

from paper_2609_20744_b200 import binding, build

N, H, HK, D = 6, 4, 2, 64


def good(lead=(N,), dtype=torch.bfloat16):
    z = lambda *s, t=dtype: torch.zeros(*s, dtype=t)
    return dict(q=z(*lead, HK, D), k=z(*lead, HK, D), v=z(*lead, H, D), beta=z(*lead, H, t=torch.float32),
                log_alpha=z(*lead, H, t=torch.float32), out=z(*lead, H, D))


def check(x, **kw):
    return binding.validate_token_args(torch.bfloat16, D, 0, x["q"], x["k"], x["v"], x["beta"], x["out"], x["log_alpha"],
                                       on_cuda=False, **kw)


def test_matching_tensors_pass():
    assert check(good()) == ((N,), H, HK, (HK * D, HK * D, H * D, H * D))
    assert check(good((3, 2)))[0] == (3, 2)
    x = good()
    x["out"] = x["log_alpha"] = None
    assert check(x)[3] == (HK * D, HK * D, H * D, H * D)


def test_slices_of_one_projected_tensor_pass_with_their_stride():
    both = torch.zeros(3, 2, 2 * HK + H, D, dtype=torch.bfloat16)
    x = good((3, 2))
    x["q"], x["k"], x["v"] = both[:, :, :HK], both[:, :, HK:2 * HK], both[:, :, 2 * HK:]
    assert check(x)[3] == ((2 * HK + H) * D,) * 3 + (H * D,)
    x["q"] = both[:, :1, :HK].expand(3, 2, HK, D)                # one token for two: not evenly spaced
    with pytest.raises(ValueError, match="q"):
        check(x)


@pytest.mark.parametrize("name,bad", [
    ("q", lambda x: x["q"].float()),
    ("q", lambda x: torch.zeros(N, 3, D, dtype=torch.bfloat16)),             # 3 key heads for 4 value heads
    ("q", lambda x: x["q"][:-1]),
    ("k", lambda x: x["k"][:, :1].contiguous()),
    ("k", lambda x: x["k"].transpose(0, 1).contiguous().transpose(0, 1)),     # heads of a token apart
    ("k", lambda x: None),
    ("v", lambda x: x["v"][..., : D // 2].contiguous()),
    ("v", lambda x: torch.zeros(N, H, D + 4, dtype=torch.bfloat16)[..., :D]),
    ("v", lambda x: torch.zeros(2 * H * D * N, dtype=torch.bfloat16).as_strided((N, H, D), (H * D + 4, D, 1))),
    ("beta", lambda x: x["beta"].bfloat16()),
    ("beta", lambda x: x["beta"][:, :1].contiguous()),
    ("log_alpha", lambda x: x["log_alpha"].double()),
    ("out", lambda x: x["out"].float()),
    ("out", lambda x: x["out"][:2]),
])
def test_mismatched_tensor_is_refused(name, bad):
    x = good()
    x[name] = bad(x)
    with pytest.raises(ValueError, match=name):
        check(x)


def test_rotary_tables():
    f, a = binding.rotary_tables((2, 1, 3), theta=100.0)
    assert a.tolist() == [0, 0, 1, 2, 2, 2] and a.dtype == torch.int32 and f.dtype == torch.float64
    assert f.tolist() == pytest.approx([1, 0.1, 1, 1, 100 ** (-1 / 3), 100 ** (-2 / 3)])
    assert binding.rotary_tables((2, 1, 1), 16.0, shared_ladder=True)[0].tolist() == pytest.approx([1, 0.5, 0.25, 0.125])
    for bad in ((1, 2), (0, 0, 0), (1, -1, 2), (1, 0.5, 1)):
        with pytest.raises(ValueError):
            binding.rotary_tables(bad)


def test_null_handle():
    build.build()
    lib = binding.load_library()
    t = binding.VdnTokenParams(ctypes.sizeof(binding.VdnTokenParams), 1, 1, 1)
    r = binding.VdnRotaryParams(ctypes.sizeof(binding.VdnRotaryParams))
    assert lib.vdn_vda_token_scan(None, None, None, None, None, None, 0, ctypes.byref(t), None, 0, None) == 1
    assert lib.vdn_vda_token_step(None, None, None, None, None, None, 0, 1, ctypes.byref(t), None) == 1
    assert lib.vdn_vda_rotate(None, None, None, None, None, 1, 1, 1, 1, 64, ctypes.byref(r), None) == 1
    assert lib.vdn_vda_token_scan_workspace_bytes(None, 10, ctypes.byref(t)) == 0


def test_struct_sizes_match_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "vdn_vda.h"\nint main(void){printf("%zu %zu", sizeof(vdn_vda_token_params), '
                   'sizeof(vdn_vda_rotary_params)); return 0;}\n')
    subprocess.run(["gcc", "-std=c99", f"-I{root}/include", str(src), "-o", str(tmp_path / "s")], check=True)
    got = subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in got] == [ctypes.sizeof(binding.VdnTokenParams), ctypes.sizeof(binding.VdnRotaryParams)]
    assert [int(x) for x in got] == [binding._TOKEN_PARAMS.size, binding._ROTARY_PARAMS.size]


def test_packed_structs_have_the_fields_of_the_structures():
    for cls, packed in ((binding.VdnTokenParams, binding._TOKEN_PARAMS), (binding.VdnRotaryParams, binding._ROTARY_PARAMS)):
        values = [1.5 if t is ctypes.c_float else i + 1 for i, (_, t) in enumerate(cls._fields_)]
        x = cls.from_buffer_copy(packed.pack(*values))
        assert [getattr(x, n) for n, _ in cls._fields_] == values
