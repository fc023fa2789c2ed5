"""What fdg_gn_* and fdg_ckpt_* refuse, and how much scratch they ask for, answered without a GPU: every refusal comes before
the first launch, and no pointer of these calls is looked at on the host."""
import ctypes as C

import pytest

from paper_1906_09108_b200 import binding as B
from paper_1906_09108_b200 import build as fdg_build

INVALID, SMALL = 1, 2
P = C.c_void_p(4096)                     # any address: aligned, never read


@pytest.fixture(scope="module")
def lib():
    fdg_build.build()
    return B.load_library()


def _scratch(lib, prec, *shape, backward=1):
    n, s = C.c_size_t(), B.fdg_gn_shape(*shape)
    rc = lib.fdg_gn_scratch_bytes(prec, C.byref(s), backward, C.byref(n))
    return rc, n.value


@pytest.mark.parametrize("prec", [B.FDG_FP32_CUDACORE, B.FDG_BF16_TC])
def test_scratch(lib, prec):
    rc, small = _scratch(lib, prec, 8, 256, 8, 4)
    assert rc == 0 and 8 * 2 * 8 * 4 <= small <= 65536           # a row of sums per CTA
    assert _scratch(lib, prec, 8, 256, 8, 4, backward=0) == (0, 0)
    for backward in (0, 1):
        rc, large = _scratch(lib, prec, 8, 65536, 128, 32, backward=backward)
        assert rc == 0 and 0 < large < 8 * 65536 * 128 * 2 // 20      # sums of chunks: a small part of the tensor
    for bad in ((0, 4, 8, 4), (4, 0, 8, 4), (4, 4, 0, 1), (4, 4, 8, 0), (4, 4, 8, 3), (4, 4, 8, 16), (-1, 4, 8, 4),
                (2 ** 31 - 1, 2 ** 31 - 1, 1024, 4), (1, 1, 2 ** 16 + 1, 1), (2 ** 20, 2 ** 19, 1, 1), (2 ** 30 + 1, 1, 1, 1)):
        assert _scratch(lib, prec, *bad)[0] == INVALID and _scratch(lib, prec, *bad, backward=0)[0] == INVALID, bad
    assert _scratch(lib, 7, 8, 256, 8, 4)[0] == INVALID
    s = B.fdg_gn_shape(8, 256, 8, 4)
    assert lib.fdg_gn_scratch_bytes(prec, None, 1, C.byref(C.c_size_t())) == INVALID
    assert lib.fdg_gn_scratch_bytes(prec, C.byref(s), 1, None) == INVALID


def test_gn_forward_refusals(lib):
    s = B.fdg_gn_shape(8, 65536, 128, 4)                       # large enough to need scratch
    need = _scratch(lib, B.FDG_BF16_TC, 8, 65536, 128, 4, backward=0)[1]
    good = dict(precision=B.FDG_BF16_TC, shape=C.byref(s), x=P, gamma=P, beta=P, res=None, act=B.FDG_ACT_RELU, eps=1e-5, y=P, stats=P,
                gate=None, codes=None, scales=None, scratch=P, bytes=need, stream=None)

    def call(**kw):
        assert set(kw) <= set(good) and kw
        return lib.fdg_gn_forward(*dict(good, **kw).values())

    for name in ("shape", "x", "gamma", "beta", "y", "stats"):
        assert call(**{name: None}) == INVALID, name
    assert call(precision=5) == INVALID and call(act=3) == INVALID and call(act=-1) == INVALID
    for eps in (0.0, -1.0, float("nan")):
        assert call(eps=eps) == INVALID
    assert call(codes=P) == INVALID and call(scales=P) == INVALID
    assert call(gate=P, act=B.FDG_ACT_NONE) == INVALID and call(gate=P, act=B.FDG_ACT_SILU) == INVALID
    assert call(res=P, act=B.FDG_ACT_SILU) == INVALID
    assert call(scratch=None) == SMALL and call(bytes=need - 1) == SMALL
    assert call(scratch=C.c_void_p(4096 + 128)) == INVALID
    for name in ("x", "y", "res"):
        assert call(**{name: C.c_void_p(4097)}) == INVALID, name
    assert call(shape=C.byref(B.fdg_gn_shape(8, 256, 9, 4))) == INVALID


def test_gn_backward_refusals(lib):
    s = B.fdg_gn_shape(8, 256, 8, 4)
    need = _scratch(lib, B.FDG_BF16_TC, 8, 256, 8, 4)[1]
    good = dict(precision=B.FDG_BF16_TC, shape=C.byref(s), dy=P, x=P, codes=None, scales=None, stats=P, gamma=P, beta=None,
                act=B.FDG_ACT_RELU, mask=P, gate=None, res=None, dx=P, dgamma=P, dbeta=P, scratch=P, bytes=need, stream=None)

    def call(**kw):
        assert set(kw) <= set(good) and kw
        return lib.fdg_gn_backward(*dict(good, **kw).values())

    for name in ("shape", "dy", "x", "stats", "gamma", "dx", "dgamma", "dbeta"):
        assert call(**{name: None}) == INVALID, name
    assert call(precision=-1) == INVALID and call(act=9) == INVALID
    assert call(codes=P, scales=P) == INVALID                                   # x as well
    assert call(x=None, codes=P) == INVALID and call(x=None, scales=P) == INVALID
    assert call(mask=None) == INVALID and call(gate=P) == INVALID               # neither gate, both
    for act in (B.FDG_ACT_NONE, B.FDG_ACT_SILU):
        assert call(act=act, beta=P) == INVALID                                 # a gate where there is none
        assert call(act=act, beta=P, mask=None, gate=P) == INVALID
    assert call(act=B.FDG_ACT_SILU, mask=None) == INVALID                       # SiLU needs beta
    assert call(scratch=None) == SMALL and call(bytes=0) == SMALL
    for name in ("dy", "x", "mask", "res", "dx"):
        assert call(**{name: C.c_void_p(4097)}) == INVALID, name


def test_ckpt_refusals(lib):
    for prec in (B.FDG_FP32_CUDACORE, B.FDG_BF16_TC):
        for rows, c in ((0, 8), (4, 0), (4, -1), (1 << 41, 8), ((1 << 33) + 1, 8), (1, (1 << 28) + 1)):
            assert lib.fdg_ckpt_encode(prec, P, rows, c, P, P, None) == INVALID
            assert lib.fdg_ckpt_decode(prec, P, P, rows, c, P, None) == INVALID
        for args in ((None, 4, 8, P, P), (P, 4, 8, None, P), (P, 4, 8, P, None), (C.c_void_p(4097), 4, 8, P, P)):
            assert lib.fdg_ckpt_encode(prec, *args, None) == INVALID
        for args in ((None, P, 4, 8, P), (P, None, 4, 8, P), (P, P, 4, 8, None), (P, P, 4, 8, C.c_void_p(4097))):
            assert lib.fdg_ckpt_decode(prec, *args, None) == INVALID
    assert lib.fdg_ckpt_encode(2, P, 4, 8, P, P, None) == INVALID
    assert lib.fdg_ckpt_decode(2, P, P, 4, 8, P, None) == INVALID


@pytest.mark.parametrize("prec", [B.FDG_FP32_CUDACORE, B.FDG_BF16_TC])
def test_shapes_up_to_the_limits_that_are_named(lib, prec):
    """2^36 values, 2^30 images, 65536 channels: nothing within these is refused for the size of a grid."""
    for shape in ((1 << 20, 1, 4104, 4104), (1 << 20, 1, 65536, 65536), (1 << 20, 1, 65536, 1), (1 << 30, 1, 64, 64), (1 << 30, 64, 1, 1), (1, 2 ** 31 - 1, 32, 4),
                  (1 << 19, 2, 65536, 65536), (16, 1 << 16, 65536, 65536), (1 << 14, 100, 4104, 8)):
        assert shape[0] * shape[1] * shape[2] <= 1 << 36
        for backward in (0, 1):
            rc, need = _scratch(lib, prec, *shape, backward=backward)
            assert rc == 0 and need % 256 == 0, (shape, backward)


def test_gn_refuses_fp32_arrays_off_their_alignment(lib):
    """A kernel reads and writes them as floats: an address that is no multiple of 4 must not reach one."""
    s = B.fdg_gn_shape(8, 256, 8, 4)
    need = _scratch(lib, B.FDG_BF16_TC, 8, 256, 8, 4)[1]
    for off in (1, 2, 3):
        odd = C.c_void_p(4096 + off)
        for name in ("gamma", "beta", "stats"):
            a = dict(x=P, gamma=P, beta=P, res=None, act=B.FDG_ACT_SILU, eps=1e-5, y=P, stats=P, gate=None, codes=None, scales=None, scratch=P)
            assert lib.fdg_gn_forward(B.FDG_BF16_TC, C.byref(s), *dict(a, **{name: odd}).values(), need, None) == INVALID, name
        for name in ("stats", "gamma", "beta", "dgamma", "dbeta"):
            a = dict(dy=P, x=P, codes=None, scales=None, stats=P, gamma=P, beta=P, act=B.FDG_ACT_SILU, mask=None, gate=None, res=None, dx=P, dgamma=P, dbeta=P,
                     scratch=P)
            assert lib.fdg_gn_backward(B.FDG_BF16_TC, C.byref(s), *dict(a, **{name: odd}).values(), need, None) == INVALID, name


def test_the_binding_takes_whole_numbers_of_groups_only(lib):
    """Also where the same shape was taken before with a number that compares equal."""
    import torch
    ew = B.EwOps(B.FDG_BF16_TC)
    shape = torch.Size((2, 4, 16))
    for groups in (4.0, "4", None):
        with pytest.raises(B.FDGError):
            ew._gn(shape, groups, 0)
    ew._gn(shape, 4, 0)
    for groups in (4.0, torch.tensor(4)):
        with pytest.raises(B.FDGError):
            ew._gn(shape, groups, 0)
