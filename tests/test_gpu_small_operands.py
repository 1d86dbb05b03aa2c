"""Operands read element by element (gates, offsets, indices, tables, lse) whose address is no multiple of their elements' size are refused on
the host.  The calls are empty, or wrong in another way that is looked at later, so that nothing runs on the GPU whatever the answer."""
import pytest
import torch

from paper_2609_20744_b200 import binding, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    binding.load_library()


def test_addresses_inside_an_element():
    vda = binding.Vda(128, "bf16")
    lib, h = vda.lib, vda.h
    t = torch.zeros(4096, device="cuda:0")
    p = t.data_ptr()
    before = t.clone()

    def refused(f, *args):
        assert f(h, *args) == 1 and b"aligned to their elements" in lib.vdn_vda_last_error(h)

    def passes(f, *args):
        assert f(h, *args) == 0 and vda.launch_count() == 0

    def cross(cu=0, lens=0, lse=0):
        return binding._CROSS_PARAMS.pack(binding._CROSS_PARAMS.size, 1, 2, 1, 1.0, 0, cu, lens, 0, lse, 0, 0, 0, 0)

    x = (p, p + 4096, p + 4096, p + 8192, 0, 5)
    for good, bad in ((cross(lse=p + 12), cross(lse=p + 2)), (cross(cu=p + 4), cross(cu=p + 1)), (cross(lens=p + 8), cross(lens=p + 6))):
        passes(lib.vdn_vda_cross_attention, *x, good, 0, 0, None)
        refused(lib.vdn_vda_cross_attention, *x, bad, 0, 0, None)

    def token(cu=0, index=0, log_alpha=0, state=0, slots=0):
        return binding._TOKEN_PARAMS.pack(binding._TOKEN_PARAMS.size, 2, 1, 0 if slots else 1, 1.0, 0.0, cu, index, log_alpha, 0, state, slots, 0, 0, 0, 0)

    x = (p, p + 4096, p + 4096, p + 1024, p + 8192, 0)
    for bad in (token(cu=p + 2), token(log_alpha=p + 3)):
        refused(lib.vdn_vda_token_scan, *x, bad, 0, 0, None)
    refused(lib.vdn_vda_token_scan, p, p + 4096, p + 4096, p + 1025, p + 8192, 0, token(), 0, 0, None)
    passes(lib.vdn_vda_token_step, *x, 1, token(index=p + 4, state=p, slots=1), None)
    refused(lib.vdn_vda_token_step, *x, 1, token(index=p + 5, state=p, slots=1), None)

    def rotary(freq=p, axis=p, positions=0, qw=0, kw=0):
        return binding._ROTARY_PARAMS.pack(binding._ROTARY_PARAMS.size, 0, 4, 1, 1, 1, 0, 0.0, freq, axis, positions, qw, kw, 0, 0, 0, 0)

    x = (p, p + 4096, p, p + 4096, 0, 1, 1, 1, 128)
    for bad in (rotary(freq=p + 4), rotary(axis=p + 2), rotary(positions=p + 1), rotary(qw=p + 2), rotary(kw=p + 2)):
        refused(lib.vdn_vda_rotate, *x, bad, None)
    assert lib.vdn_vda_rotate(h, *x, rotary(), None) == 1 and b"positive" in lib.vdn_vda_last_error(h)          # (B = 0)
    torch.cuda.synchronize()
    assert t.equal(before) and vda.status() == binding.VDN_OK
