"""Group norm with an activation and tensors held in 8 bits (fdg_gn_*, fdg_ckpt_*) through the C ABI, against their definitions in
float64 (oracle/norms.py) on the same inputs.

Tolerances, element by element.  A stored value is rounded to nearest: half a step, 2^-8 (bf16) or 2^-24 (fp32) of the value.
Everything before is fp32 with sums whose longest chain (a thread's values, its row of threads, the lanes of a group) is
under 256 terms, so a sum is off by less than 256 * 2^-24 of the sum of its terms' magnitudes (K below); means, spreads and the
two group sums of the backward pass enter an output at most once each with a factor of at most 1 (SiLU's slope: 1.1), and the
few operations around them are below that.  The magnitude that K multiplies is that of the terms, before any cancellation:
(|x| + |mean|)*rstd stands for |xhat|.  Checkpoints have no tolerance: the format leaves no freedom."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import norms as L

pytestmark = pytest.mark.gpu
EPS = 1e-5
K = 256 * 2.0 ** -24
PRECISIONS = ["fp32", "bf16"]

# (N, pixels, C, groups)
SHAPES = [
    (1, 1, 1, 1), (3, 1, 8, 4), (2, 1, 30, 5), (5, 4, 2, 2),        # one pixel, one value, groups of a few values
    (8, 256, 8, 4), (4, 1024, 16, 4), (3, 64, 64, 64),              # narrow layers; a group per channel
    (2, 1024, 160, 32), (2, 64, 640, 1), (3, 49, 320, 32),          # groups of 5 channels; one group; odd maps
    (2, 784, 30, 6), (3, 65, 33, 11), (7, 9, 24, 3), (1, 100, 7, 7),   # channels that fill no column
    (2, 17, 2048, 16), (1, 3, 2056, 8), (2, 5, 4104, 27), (1, 2, 4112, 1),      # as wide as a CTA goes, and wider
    (1, 3, 65536, 32), (1, 2, 65536, 65536), (500, 5, 16, 4), (700, 2, 30, 3),     # the widest; more images than CTAs run at once
]
# images that no cluster holds
LARGE = [(1, 16384, 64, 8), (2, 9001, 160, 32), (1, 20011, 30, 1)]


def _ops(prec_name):
    from paper_1906_09108_b200 import binding as B
    return B, B.EwOps(B.FDG_BF16_TC if prec_name == "bf16" else B.FDG_FP32_CUDACORE)


def _half_step(dtype):
    return torch.finfo(dtype).eps / 2


def _mk(shape, seed, dtype, scale=1.0, shift=0.0):
    a = np.random.default_rng(seed).standard_normal(shape) * scale + shift
    t = torch.from_numpy(a.astype(np.float32)).cuda().to(dtype)
    return t, t.double().cpu().numpy()


def _f32(a):
    return torch.from_numpy(np.asarray(a, np.float32)).cuda()


def _np(t):
    return t.double().cpu().numpy()


def _near(got, want, tol, what=""):
    got = _np(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(np.abs(got - want)[bad].max()), float(np.broadcast_to(tol, want.shape)[bad].min()))


def _params(c, seed):
    r = np.random.default_rng(seed)
    return ((1 + 0.3 * r.standard_normal(c)).astype(np.float32).astype(np.float64),
            (0.2 * r.standard_normal(c)).astype(np.float32).astype(np.float64))



def _channels(a, c):
    """[N, groups] -> [N, 1, c]."""
    return np.repeat(a, c // a.shape[1], 1)[:, None, :]


def _size(xo, stats, c):
    """What stands for |xhat|: (|x| + |mean|) * rstd."""
    return (np.abs(xo) + np.abs(_channels(stats[0], c))) * _channels(stats[1], c)


def _check_forward(ew, shape, act, with_res, seed=0, scale=1.3, shift=0.4, gate=False, ckpt=False, x=None):
    n, p, c, groups = shape
    if x is None:
        x, xo = _mk((n, p, c), seed + 1, ew.dtype, scale, shift)
    else:
        xo = _np(x)
    res, reso = _mk((n, p, c), seed + 2, ew.dtype) if with_res else (None, None)
    gamma, beta = _params(c, seed + 3)
    y, stats, bits, held = ew.gn_forward(x, groups, _f32(gamma), _f32(beta), act=act, res=res, eps=EPS, gate=gate, checkpoint=ckpt)
    yo, z, st = L.groupnorm_forward(xo, groups, gamma, beta, EPS, act, reso)
    # the mean: K of the mean magnitude; rstd: its square root halves the spread's error, and the CTAs' means enter squared
    mag = np.abs(xo).reshape(n, p, groups, -1).mean((1, 3))
    _near(stats[0], st[0], K * mag + 1e-30, "mean")
    _near(stats[1], st[1], st[1] * (K + (K * mag * st[1]) ** 2), "rstd")
    size = _size(xo, st, c) * np.abs(gamma) + np.abs(beta) + (0 if reso is None else np.abs(reso))
    _near(y, yo, _half_step(ew.dtype) * np.abs(yo) + 1.1 * K * size, "y")
    if gate:
        b = np.unpackbits(bits.cpu().numpy(), axis=-1, bitorder="little")
        assert (b[..., :c] == (_np(y) > 0)).all() and not b[..., c:].any()
    if ckpt:
        codes, scales = L.ckpt_encode(xo.reshape(-1, c))
        assert (held[0].cpu().numpy().reshape(-1, c) == codes).all() and (held[1].cpu().numpy().reshape(n * p, -1) == scales).all()
    return x, xo, y, stats, bits, held


def _check_backward(ew, shape, act, seed, xo, x_arg, stats, y, bits, with_res, use_bits):
    """x_arg is what the call is given, xo the float64 values that it stands for."""
    n, p, c, groups = shape
    dy, dyo = _mk((n, p, c), seed + 4, ew.dtype, 0.01)
    res, reso = _mk((n, p, c), seed + 5, ew.dtype, 0.01) if with_res else (None, None)
    gamma, beta = _params(c, seed + 3)
    st = _np(stats)
    kw = dict(mask=None, gate=None)
    if act == "relu":
        kw = dict(mask=None, gate=bits) if use_bits else dict(mask=y, gate=None)
    dx, dgamma, dbeta = ew.gn_backward(dy, x_arg, stats, groups, _f32(gamma), _f32(beta), act=act, res=res, **kw)
    xhat = L.groupnorm_xhat(xo, st, groups)
    size = _size(xo, st, c)
    dz = dyo * ((_np(y) > 0) if act == "relu" else L.activation_slope(gamma * xhat + beta, act))
    # SiLU: its slope moves by at most half of what z moves
    adz = np.abs(dz) + (0.5 * np.abs(dyo) * (size * np.abs(gamma) + np.abs(beta)) if act == "silu" else 0)
    dxo, dgo, dbo = L.groupnorm_backward(dz, xo, st, groups, gamma, reso)
    mean = lambda t: _channels(t.reshape(n, p, groups, -1).mean((1, 3)), c)  # noqa: E731
    h = adz * np.abs(gamma)
    mag = _channels(st[1], c) * (h + mean(h) + size * mean(h * size)) + (0 if reso is None else np.abs(reso))
    _near(dx, dxo, _half_step(ew.dtype) * np.abs(dxo) + 2 * K * mag, "dx")
    _near(dgamma, dgo, 2 * K * (adz * size).sum((0, 1)) + 1e-30, "dgamma")
    _near(dbeta, dbo, 2 * K * adz.sum((0, 1)) + 1e-30, "dbeta")
    return dx, dgamma, dbeta


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("shape", SHAPES + LARGE, ids=str)
def test_forward(prec_name, shape):
    _, ew = _ops(prec_name)
    _check_forward(ew, shape, "none", False)
    _check_forward(ew, shape, "relu", True, seed=10, gate=True, ckpt=shape[0] * shape[1] * shape[2] < 200000)
    _check_forward(ew, shape, "silu", False, seed=20)


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("shape", SHAPES + LARGE, ids=str)
def test_backward(prec_name, shape):
    _, ew = _ops(prec_name)
    n, p, c, groups = shape
    for seed, act in ((30, "none"), (40, "relu"), (50, "silu")):
        x, xo, y, stats, bits, held = _check_forward(ew, shape, act, False, seed=seed, gate=act == "relu")
        _check_backward(ew, shape, act, seed, xo, x, stats, y, bits, act == "none", False)
        held = ew.ckpt_encode(x)
        heldo = L.ckpt_decode(held[0].cpu().numpy().reshape(-1, c), held[1].cpu().numpy().reshape(n * p, -1)).reshape(n, p, c)
        _check_backward(ew, shape, act, seed, heldo, held, stats, y, bits, True, True)


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("by", [1, 2, 4])
@pytest.mark.parametrize("shape", [(2, 40, 16, 4), (2, 24, 64, 2), (2, 9, 30, 5), (2, 33, 20, 5), (3, 7, 12, 4), (1, 16384, 64, 8),
                                   (1, 20000, 36, 4)], ids=str)
def test_any_alignment(prec_name, shape, by):
    """Contiguous tensors that start `by` elements off a vector's alignment."""
    B, ew = _ops(prec_name)
    n, p, c, groups = shape

    def shifted(t):
        buf = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")
        out = buf[by:].view(t.shape)
        out.copy_(t)
        return out

    x = shifted(_mk((n, p, c), 61, ew.dtype)[0])
    small = n * p * c < 200000
    x, xo, y, stats, bits, held = _check_forward(ew, shape, "relu", False, seed=60, gate=True, ckpt=small, x=x)
    _check_backward(ew, shape, "relu", 60, xo, x, stats, shifted(y), bits, True, False)
    codes, scales = (shifted(t) for t in ew.ckpt_encode(x))
    heldo = L.ckpt_decode(codes.cpu().numpy().reshape(-1, c), scales.cpu().numpy().reshape(n * p, -1)).reshape(n, p, c)
    if small:
        assert (codes.cpu().numpy() == held[0].cpu().numpy()).all()
    assert (_np(ew.ckpt_decode((codes, scales))) == heldo).all()
    _check_backward(ew, shape, "relu", 60, heldo, (codes, scales), stats, y, bits, False, True)


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("shape", [(2, 300, 40, 4), (1, 16384, 64, 8)], ids=str)
def test_offsets_of_many_spreads(prec_name, shape):
    """A mean of a thousand spreads: no difference of large sums.  The first pixel, where a pivot might be taken, is far off."""
    _, ew = _ops(prec_name)
    n, p, c, groups = shape
    x, _ = _mk((n, p, c), 71, ew.dtype, 1.0, 1000.0)
    x[:, 0] = 0.0
    _check_forward(ew, shape, "none", False, seed=70, x=x)
    x, _ = _mk((n, p, c), 72, ew.dtype, 0.0, 3.0)               # no spread at all: eps alone
    _check_forward(ew, shape, "none", False, seed=70, x=x)


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("shape", [(3, 40, 16, 4), (3, 9001, 160, 32)], ids=str)
def test_what_is_not_finite_stays_in_its_group(prec_name, shape):
    _, ew = _ops(prec_name)
    n, p, c, groups = shape
    cg = c // groups
    x, _ = _mk((n, p, c), 81, ew.dtype)
    gamma, beta = (_f32(a) for a in _params(c, 82))
    clean = ew.gn_forward(x, groups, gamma, beta, act="relu", gate=True, checkpoint=True)
    x[1, 7, 0] = float("nan")
    x[1, 8, cg] = float("inf")
    y, stats, bits, held = ew.gn_forward(x, groups, gamma, beta, act="relu", gate=True, checkpoint=True)
    assert not stats[:, 1, :2].isfinite().any()
    assert y[1, :, :2 * cg].isnan().all()
    keep = torch.ones_like(x, dtype=torch.bool)
    keep[1, :, :2 * cg] = False
    assert torch.equal(y[keep], clean[0][keep])
    others = torch.ones_like(stats, dtype=torch.bool)
    others[:, 1, :2] = False
    assert torch.equal(stats[others], clean[1][others])
    back = ew.ckpt_decode(held)
    assert back[1, 7, :min(32, c)].isnan().all() and back[1, 8, :min(32, c)].isnan().all()
    back[1, 7:9], ref = 0, ew.ckpt_decode(clean[3])
    ref[1, 7:9] = 0
    assert torch.equal(back[1, 9:], ref[1, 9:]) and torch.equal(back[0], ref[0]) and torch.equal(back[2], ref[2])
    # the backward pass: images whose own x and dy are finite are as they were; the parameters' gradients are not finite
    dy, _ = _mk((n, p, c), 83, ew.dtype)
    a = ew.gn_backward(dy, x, stats, groups, gamma, act="relu", mask=clean[0])
    b = ew.gn_backward(dy, held, stats, groups, gamma, act="relu", gate=clean[2])
    want = ew.gn_backward(dy, clean[3], clean[1], groups, gamma, act="relu", gate=clean[2])
    assert torch.equal(b[0][0], want[0][0]) and torch.equal(b[0][2], want[0][2])
    assert a[0][1].isnan().any() and a[1][:2 * cg].isnan().all() and a[1][2 * cg:].isfinite().all() and a[2].isfinite().all()


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("rows, c", [(1, 1), (5, 8), (300, 16), (70, 24), (33, 30), (64, 32), (9, 33), (50, 40), (20, 160), (6, 650), (4099, 64),
                                     (1, 1000), (40, 12), (40, 20), (33, 100), (50, 72), (9, 34)])
def test_checkpoints_are_the_format(prec_name, rows, c):
    _, ew = _ops(prec_name)
    g = np.random.default_rng(rows * 1000 + c)
    a = g.standard_normal((rows, c)) * 10.0 ** g.integers(-38, 38, (rows, 1))
    a[g.random((rows, c)) < 0.1] = 0
    x = torch.from_numpy(a.astype(np.float32)).cuda().to(ew.dtype)
    top = torch.finfo(ew.dtype).max
    if rows > 4:
        x[0] = 0
        x[1, 0] = top
        x[2, c - 1] = float("nan")
        x[3, 0] = -float("inf")
        x[4] = torch.finfo(ew.dtype).tiny
        # borders of the step: 127.5 steps and the values beside it, ties
        edge = torch.tensor([127.5, 127.0, 0.5, 1.5, -2.5, 63.75, 126.5, -127.5], dtype=ew.dtype, device="cuda")
        x[-1, :min(c, 8)] = edge[:min(c, 8)]
    codes, scales = ew.ckpt_encode(x)
    want = L.ckpt_encode(_np(x))
    assert (codes.cpu().numpy() == want[0]).all() and (scales.cpu().numpy() == want[1]).all()
    back = _np(ew.ckpt_decode((codes, scales)))
    np.testing.assert_array_equal(back, L.ckpt_decode(*want))
    again = ew.ckpt_encode(ew.ckpt_decode((codes, scales)))       # what is held is held exactly
    np.testing.assert_array_equal(_np(ew.ckpt_decode(again)), back)


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("shape", [(3, 37, 30, 5), (3, 37, 40, 5), (1, 16390, 72, 8)], ids=str)
def test_nothing_is_written_past_the_outputs(prec_name, shape):
    """Every output and the scratch stand in buffers of their own with a pattern on both sides."""
    B, ew = _ops(prec_name)
    n, p, c, groups = shape
    lib, prec = ew.lib, ew.precision
    b = 2 if prec_name == "bf16" else 4
    need, back, s = C.c_size_t(), C.c_size_t(), B.fdg_gn_shape(n, p, c, groups)
    assert lib.fdg_gn_scratch_bytes(prec, C.byref(s), 0, C.byref(need)) == 0
    assert lib.fdg_gn_scratch_bytes(prec, C.byref(s), 1, C.byref(back)) == 0
    sizes = dict(y=n * p * c * b, stats=2 * n * groups * 4, gate=n * p * -(-c // 8), codes=n * p * c, scales=n * p * -(-c // 32),
                 scratch=need.value, scratch_b=back.value, dx=n * p * c * b, dgamma=4 * c, dbeta=4 * c)
    pad = 512
    bufs = {k: torch.full((v + 2 * pad,), 0x5A, dtype=torch.uint8, device="cuda") for k, v in sizes.items()}
    at = {k: v.data_ptr() + pad for k, v in bufs.items()}
    x, dy = _mk((n, p, c), 91, ew.dtype)[0], _mk((n, p, c), 92, ew.dtype)[0]
    gamma, beta = (_f32(a) for a in _params(c, 93))
    st = torch.cuda.current_stream().cuda_stream
    assert lib.fdg_gn_forward(prec, C.byref(s), x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), None, B.FDG_ACT_RELU, EPS, at["y"],
                              at["stats"], at["gate"], at["codes"], at["scales"], at["scratch"], need.value, st) == 0
    for held in (False, True):
        assert lib.fdg_gn_backward(prec, C.byref(s), dy.data_ptr(), None if held else x.data_ptr(), at["codes"] if held else None,
                                   at["scales"] if held else None, at["stats"], gamma.data_ptr(), beta.data_ptr(), B.FDG_ACT_RELU,
                                   None if held else at["y"], at["gate"] if held else None, None, at["dx"], at["dgamma"], at["dbeta"],
                                   at["scratch_b"], back.value, st) == 0
    torch.cuda.synchronize()
    for k, v in bufs.items():
        assert (v[:pad] == 0x5A).all() and (v[pad + sizes[k]:] == 0x5A).all(), k
    y, stats, bits, kept = ew.gn_forward(x, groups, gamma, beta, act="relu", eps=EPS, gate=True, checkpoint=True)
    for name, t in (("y", y), ("stats", stats), ("gate", bits), ("codes", kept[0]), ("scales", kept[1])):
        assert torch.equal(bufs[name][pad:pad + sizes[name]], t.reshape(-1).view(torch.uint8)), name


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("shape", [(4, 1024, 160, 32), (2, 12000, 96, 8)], ids=str)
def test_same_bits_again_on_streams_and_in_graphs(prec_name, shape):
    """Two calls side by side on streams of their own, and captured and replayed on new inputs, give the bits of one call alone."""
    _, ew = _ops(prec_name)
    n, p, c, groups = shape
    gamma, beta = (_f32(a) for a in _params(c, 101))

    def both(x, dy):
        y, stats, bits, held = ew.gn_forward(x, groups, gamma, beta, act="relu", gate=True, checkpoint=True)
        return [y, stats, bits, *held, *ew.gn_backward(dy, held, stats, groups, gamma, beta, act="relu", gate=bits)]

    ins = [(_mk((n, p, c), 102 + i, ew.dtype)[0], _mk((n, p, c), 112 + i, ew.dtype)[0]) for i in range(2)]
    want = [both(*i) for i in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ins]
    for _ in range(5):
        got = []
        for s, i in zip(streams, ins):
            with torch.cuda.stream(s):
                got.append(both(*i))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, w))
    x, dy = ins[0][0].clone(), ins[0][1].clone()
    graphs = []
    for _ in range(2):                                   # two recorded graphs, replayed in turn
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = both(x, dy)
        graphs.append((g, out))
    for k in (1, 0, 1):
        x.copy_(ins[k][0])
        dy.copy_(ins[k][1])
        for g, out in graphs:
            g.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want[k]))


def test_binding_refuses_what_the_library_cannot_see():
    B, ew = _ops("bf16")
    x = torch.zeros((2, 4, 4, 16), dtype=torch.bfloat16, device="cuda")
    one, zero = torch.ones(16, device="cuda"), torch.zeros(16, device="cuda")
    y, stats, bits, held = ew.gn_forward(x, 4, one, zero, act="relu", gate=True, checkpoint=True)
    dy = torch.zeros_like(x)
    bad = [
        lambda: ew.gn_forward(x.float(), 4, one, zero),
        lambda: ew.gn_forward(x.cpu(), 4, one, zero),
        lambda: ew.gn_forward(x.transpose(1, 3), 4, one[:4], zero[:4]),
        lambda: ew.gn_forward(x, 3, one, zero),
        lambda: ew.gn_forward(x, 4, one[:8], zero),
        lambda: ew.gn_forward(x, 4, one, zero.bfloat16()),
        lambda: ew.gn_forward(x, 4, one, zero, act="gelu"),
        lambda: ew.gn_forward(x, 4, one, zero, act="silu", res=dy),
        lambda: ew.gn_forward(x, 4, one, zero, act="silu", gate=True),
        lambda: ew.gn_forward(x, 4, one, zero, res=dy[:1]),
        lambda: ew.gn_forward(x[:0], 4, one, zero),
        lambda: ew.gn_backward(dy, x, stats, 4, one, act="relu"),
        lambda: ew.gn_backward(dy, x, stats, 4, one, act="relu", mask=y, gate=bits),
        lambda: ew.gn_backward(dy, x, stats, 4, one, act="none", mask=y),
        lambda: ew.gn_backward(dy, x, stats, 4, one, act="silu"),
        lambda: ew.gn_backward(dy, x[:1], stats, 4, one),
        lambda: ew.gn_backward(dy, (held[0], held[1][:1]), stats, 4, one),
        lambda: ew.gn_backward(dy, (held[0].view(torch.uint8), held[1]), stats, 4, one),
        lambda: ew.gn_backward(dy, x, stats[:1], 4, one),
        lambda: ew.gn_backward(dy, x, stats, 4, one, act="relu", gate=bits[:1]),
        lambda: ew.ckpt_encode(x.float()),
        lambda: ew.ckpt_encode(x[..., ::2]),
        lambda: ew.ckpt_encode(x[:0]),
        lambda: ew.ckpt_decode((held[0], held[1].float())),
        lambda: ew.ckpt_decode((held[0][:1], held[1])),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(B.FDGError):
            call()
            print("not refused:", i)


def test_gradient_matches_differences():
    """The fp32 calls against central differences of the float64 forward pass."""
    _, ew = _ops("fp32")
    n, p, c, groups, h = 2, 6, 12, 3, 1e-5
    x, xo = _mk((n, p, c), 121, ew.dtype)
    dy, dyo = _mk((n, p, c), 122, ew.dtype)
    gamma, beta = _params(c, 123)
    _, stats, _, _ = ew.gn_forward(x, groups, _f32(gamma), _f32(beta), act="silu")
    grads = [_np(t) for t in ew.gn_backward(dy, x, stats, groups, _f32(gamma), _f32(beta), act="silu")]
    for which, (arg, grad) in enumerate(zip((xo, gamma, beta), grads)):
        for i in range(0, arg.size, 5):
            side = []
            for d in (-h, h):
                a = arg.copy().reshape(-1)
                a[i] += d
                args = [xo, gamma, beta]
                args[which] = a.reshape(arg.shape)
                side.append((L.groupnorm_forward(args[0], groups, args[1], args[2], EPS, "silu")[0] * dyo).sum())
            # differences are good to 1e-7 here (h^2 and 1e-16/h); fp32 to K of terms of order 10
            assert abs((side[1] - side[0]) / (2 * h) - grad.reshape(-1)[i]) <= 1e-7 + 20 * K, (which, i)


def test_offsets_past_32_bits():
    """More than 2^31 values: the last image's results, against its own definition in 64 bits (on the GPU, with the tolerances
    of the small cases) and, for what is held in 8 bits, against the image alone."""
    _, ew = _ops("bf16")
    n, p, c, groups = 17, 1 << 20, 128, 8                         # 2.28e9 values
    x = torch.empty((n, p, c), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    for i in range(n):
        x[i] = torch.randn((p, c), generator=g, device="cuda")
    gamma, beta = (_f32(a) for a in _params(c, 131))
    y, stats, bits, held = ew.gn_forward(x, groups, gamma, beta, act="relu", gate=True, checkpoint=True)

    def by_group(t):
        return t.view(p, groups, c // groups)

    xl = x[-1].double()
    mean = by_group(xl).mean((0, 2))
    rstd = 1 / ((by_group(xl) - mean[:, None]).square().mean((0, 2)) + EPS).sqrt()
    wide = lambda t: t.repeat_interleave(c // groups)  # noqa: E731
    assert ((stats[0, -1] - mean).abs() <= K * by_group(xl.abs()).mean((0, 2))).all() and ((stats[1, -1] - rstd).abs() <= K * rstd).all()
    want = ((xl - wide(mean)) * wide(rstd) * gamma + beta).clamp(min=0)
    size = (xl.abs() + wide(mean).abs()) * wide(rstd)
    assert ((y[-1].double() - want).abs() <= _half_step(ew.dtype) * want + 1.1 * K * (size * gamma.abs() + beta.abs())).all()
    assert torch.equal((bits[-1].unsqueeze(-1) >> torch.arange(8, device="cuda", dtype=torch.uint8)).bitwise_and(1).view(p, c) != 0, y[-1] > 0)
    alone = ew.ckpt_encode(x[-1:].clone())
    apart = ew.ckpt_encode(x)
    for a in (held, apart):
        assert torch.equal(a[0][-1:], alone[0]) and torch.equal(a[1][-1:], alone[1])
    del apart, want, size
    back = ew.ckpt_decode(held)[-1]
    assert torch.equal(back, ew.ckpt_decode(alone)[0])
    dx = ew.gn_backward(y, held, stats, groups, gamma, act="relu", gate=bits)[0][-1].double()
    m, r = (wide(stats[i, -1].double()) for i in range(2))
    xhat, h = (back.double() - m) * r, y[-1].double() * gamma
    one, two = by_group(h).mean((0, 2)), by_group(h * xhat).mean((0, 2))
    want = r * (h - wide(one) - xhat * wide(two))
    size = (back.double().abs() + m.abs()) * r
    mag = r * (h.abs() + wide(by_group(h.abs()).mean((0, 2))) + size * wide(by_group(h.abs() * size).mean((0, 2))))
    assert ((dx - want).abs() <= _half_step(ew.dtype) * want.abs() + 2 * K * mag).all()


@pytest.mark.parametrize("c, groups", [(32, 4), (160, 32)])
def test_a_block_with_its_activations_held_in_8_bits(c, groups):
    """The operators as a residual branch uses them: conv -> group norm + ReLU -> conv forward, keeping x and the ReLU's output
    in 8 bits and the gate in bits, and back: data gradient, group norm from the checkpoint, weight gradients from decoded
    checkpoints.  Each step against its float64 definition on the step's own inputs."""
    B, ew = _ops("bf16")
    conv = B.ConvOps(B.FDG_BF16_TC)
    n, h, w = 4, 16, 16
    s = B.fdg_conv_shape(n, h, w, c, c, 3, 1, 1)
    x0 = _mk((n, h, w, c), 141, ew.dtype)[0]
    w1, w2 = (_mk((c, 3, 3, c), 142 + i, ew.dtype, (2 / (9 * c)) ** 0.5)[0] for i in range(2))
    gamma, beta = _params(c, 144)
    x1 = conv.forward(s, x0, w1)
    y1, stats, bits, held1 = ew.gn_forward(x1, groups, _f32(gamma), _f32(beta), act="relu", gate=True, checkpoint=True)
    held_y = ew.ckpt_encode(y1)
    dy2 = _mk((n, h, w, c), 145, ew.dtype, 0.1)[0]

    yo, _, st = L.groupnorm_forward(_np(x1).reshape(n, h * w, c), groups, gamma, beta, EPS, "relu")
    assert np.abs(_np(y1).reshape(yo.shape) - yo).max() <= _half_step(ew.dtype) * np.abs(yo).max() + 16 * K
    # weight gradient of the second convolution: its input as held, which bf16 holds exactly
    y1h = ew.ckpt_decode(held_y)
    assert torch.equal(y1h.float(), held_y[0].float() * (held_y[1].int() << 23).view(torch.float32).repeat_interleave(32, -1)[..., :c])
    dw2 = conv.wgrad(s, y1h, dy2)
    ref = torch.nn.grad.conv2d_weight(y1h.double().permute(0, 3, 1, 2), (c, c, 3, 3), dy2.double().permute(0, 3, 1, 2), padding=1).permute(0, 2, 3, 1)
    assert float((dw2.double() - ref).norm() / ref.norm()) <= 1e-5
    # against the tensor itself: dy is independent of what the 8 bits left out, so the weight gradient is as far off as they are
    full = conv.wgrad(s, y1, dy2)
    assert float((dw2 - full).norm() / full.norm()) <= 2 * float((y1h.float() - y1.float()).norm() / y1.float().norm())
    dy1 = conv.dgrad(s, dy2, w2, conv.flip_weights(s, w2))
    dx1, dgamma, dbeta = ew.gn_backward(dy1, held1, stats, groups, _f32(gamma), act="relu", gate=bits)
    heldo = L.ckpt_decode(held1[0].cpu().numpy().reshape(-1, c), held1[1].cpu().numpy().reshape(n * h * w, -1)).reshape(n, h * w, c)
    dz = _np(dy1).reshape(n, h * w, c) * (_np(y1).reshape(n, h * w, c) > 0)
    dxo, dgo, dbo = L.groupnorm_backward(dz, heldo, _np(stats), groups, gamma)
    for got, want in ((dx1.reshape(n, h * w, c), dxo), (dgamma, dgo), (dbeta, dbo)):
        assert np.abs(_np(got) - want).max() <= (_half_step(ew.dtype) + 4 * K) * np.abs(want).max()
    exact = ew.gn_backward(dy1, x1, stats, groups, _f32(gamma), act="relu", mask=y1)
    off = float((ew.ckpt_decode(held1).float() - x1.float()).norm() / x1.float().norm())
    for got, want in zip((dx1, dgamma, dbeta), exact):
        assert float((got.float() - want.float()).norm() / want.float().norm()) <= 2 * off + _half_step(ew.dtype)
    assert not conv.timed_out()


@pytest.mark.parametrize("prec_name", PRECISIONS)
def test_silu_over_its_range(prec_name):
    """gamma = 0 and one pixel make z = beta exactly, dbeta = SiLU's slope there.  u = 2^-24.  A sigmoid s is off by d of itself: fp32
    storage 4u (expf, 2 ulp) + u (1 + exp) + u (the reciprocal); 16-bit storage (1 + 1)|z|u (z*log2(e): the constant and the product)
    + 4u (the exponential) + u + 4u (the product of two denominators, its reciprocal at 1 ulp, the product that gives one back).
    z*s adds u; s*(1 + z(1 - s)) adds |z|(d*s + 2u(1 - s) + u) + u inside the bracket and d + u outside.  fp32: a sigmoid below the
    smallest normal number, 2^-126, may be 0, which costs up to 2^-126 (1 + |z|)."""
    _, ew = _ops(prec_name)
    dt = ew.dtype
    c = 4096
    z = np.linspace(-120, 120, c) if prec_name == "fp32" else np.linspace(-40, 40, c)
    z = z.astype(np.float32)
    zz = z.astype(np.float64)
    x = torch.zeros(1, 1, c, device="cuda", dtype=dt)
    zero = torch.zeros(c, device="cuda")
    u = 2.0 ** -24
    s = 1 / (1 + np.exp(-zz))
    d = 6 * u if prec_name == "fp32" else (2 * np.abs(zz) + 9) * u
    lost = 2.0 ** -126 * (1 + np.abs(zz))
    y, stats, _, _ = ew.gn_forward(x, 4, zero, _f32(z), act="silu")
    _near(y.reshape(c), zz * s, np.abs(zz * s) * (_half_step(dt) * (1 + 2 * d) + d + u) + lost, "y")
    _, _, db = ew.gn_backward(torch.ones_like(x), x, stats, 4, zero, _f32(z), act="silu")
    slope = s * (1 + zz * (1 - s))
    inner = np.abs(zz) * (d * s + 2 * u * (1 - s) + u) + u
    _near(db, slope, s * inner * (1 + 2 * d) + np.abs(slope) * (d + u) + lost, "dbeta")
    # past both ends, and nothing there: the ends of the formula as a division gives them
    ends = _f32([0.0, -1e4, 1e4, -3e38, 3e38, float("inf"), float("nan"), 1.0])
    y = ew.gn_forward(x[..., :8].contiguous(), 4, zero[:8], ends, act="silu")[0].reshape(8).float().cpu()
    if prec_name == "fp32":
        assert y[1] == 0 and y[3] == 0
    assert y[0] == 0 and y[2] == ends[2].to(dt).float() and y[5] == float("inf") and torch.isnan(y[6]) and torch.isfinite(y[7])


# many small images: a few rows of threads each, several to a CTA, more than run at once; groups inside and across columns
SMALL = [
    (4096, 4, 64, 4), (2000, 9, 128, 32), (2000, 1, 512, 32), (900, 3, 30, 6), (1300, 7, 33, 11), (601, 21, 160, 32), (3001, 2, 8, 1),
    (500, 200, 3, 1), (700, 5, 264, 3), (450, 2, 2048, 16), (450, 3, 1000, 1), (500, 1, 2048, 2048), (2999, 1, 1, 1), (150, 90, 40, 40),
    (450, 5, 640, 8), (20011, 1, 48, 2), (300, 100, 64, 8), (1100, 25, 96, 4), (800, 6, 20, 5),
    # rows in slices, and where groups allow none
    (300, 1, 4096, 32), (40, 3, 5120, 16), (16, 130, 256, 8), (33, 49, 512, 32), (200, 2, 4096, 1), (20, 2, 6144, 64), (700, 1, 2176, 2),
]


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("shape", SMALL, ids=str)
def test_many_small_images(prec_name, shape):
    _, ew = _ops(prec_name)
    c = shape[2]
    for seed, act, gate in ((60, "relu", True), (65, "silu", False)):
        x, xo, y, stats, bits, held = _check_forward(ew, shape, act, gate, seed=seed, gate=gate, ckpt=True)
        kept = L.ckpt_decode(held[0].cpu().numpy().reshape(-1, c), held[1].cpu().numpy().reshape(shape[0] * shape[1], -1)).reshape(xo.shape)
        _check_backward(ew, shape, act, seed, kept, held, stats, y, bits, gate, gate)
    for seed, act in ((70, "none"), (80, "relu"), (90, "silu")):
        x, xo, y, stats, bits, held = _check_forward(ew, shape, act, False, seed=seed, gate=act == "relu")
        _check_backward(ew, shape, act, seed, xo, x, stats, y, bits, act == "none", False)


@pytest.mark.parametrize("prec_name", PRECISIONS)
def test_small_images_far_from_zero_and_not_finite(prec_name):
    """The variance of values far from zero, and one image with an infinity and one with a NaN: only these are lost."""
    _, ew = _ops(prec_name)
    n, p, c, groups = 700, 9, 64, 4
    x, xo = _mk((n, p, c), 3, ew.dtype, 1.0, 300.0)
    x[5, 3, 7], x[600, 0, 63] = float("inf"), float("nan")
    xo = x.double().cpu().numpy()
    gamma, beta = _params(c, 4)
    y, stats, _, held = ew.gn_forward(x, groups, _f32(gamma), _f32(beta), act="silu", checkpoint=True)
    lost = np.zeros((n, groups), bool)
    lost[5, 0] = lost[600, 3] = True
    st = _np(stats)
    assert np.isnan(st[0][600, 3]) and not np.isfinite(st[0][5, 0]) and np.isfinite(st[:, ~lost]).all()
    back = _np(ew.ckpt_decode(held))
    clean = [i for i in range(n) if i not in (5, 600)]
    want = L.groupnorm_stats(xo[clean], groups, EPS)
    mag = np.abs(xo[clean]).reshape(len(clean), p, groups, -1).mean((1, 3))
    _near(st[0][clean], want[0], K * mag, "mean")
    _near(st[1][clean], want[1], want[1] * (K + (K * mag * want[1]) ** 2), "rstd")
    assert np.isfinite(_np(y)[clean]).all() and np.isfinite(back[clean]).all()
    yl = np.isnan(_np(y).reshape(n, p, groups, -1)).all((1, 3))
    assert yl[600, 3] and yl[5, 0] and yl.sum() == 2


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("shape", [(2000, 4, 64, 4), (700, 1, 4096, 32)], ids=str)
def test_small_images_captured_and_beside_one_another(prec_name, shape):
    """The same bits from a graph that is replayed on new values, and from calls on two streams at once."""
    _, ew = _ops(prec_name)
    n, p, c, groups = shape
    gamma, beta = (_f32(t) for t in _params(c, 5))
    sets = [(_mk((n, p, c), 6 + i, ew.dtype)[0], _mk((n, p, c), 16 + i, ew.dtype, 0.01)[0]) for i in range(3)]

    def step(x, dy):
        y, stats, bits, held = ew.gn_forward(x, groups, gamma, beta, act="relu", gate=True, checkpoint=True)
        return (y, stats, bits, *held, *ew.gn_backward(dy, held, stats, groups, gamma, act="relu", gate=bits))

    want = [step(*s) for s in sets]
    torch.cuda.synchronize()
    x, dy = sets[0][0].clone(), sets[0][1].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(x, dy)
    for (a, b), w in zip(sets, want):
        x.copy_(a)
        dy.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, u) for t, u in zip(got, w))
    streams = [torch.cuda.Stream() for _ in sets]
    beside = []
    for _ in range(4):
        for st, s in zip(streams, sets):
            with torch.cuda.stream(st):
                beside.append(step(*s))
    torch.cuda.synchronize()
    for i, b in enumerate(beside):
        assert all(torch.equal(t, u) for t, u in zip(b, want[i % 3]))


# ---- long threads, blank groups, far tails, options together ------------------------------------------------------------

def _stats64(x, groups):
    """mean, rstd [N, groups] of a tensor on the GPU, in float64, image by image."""
    n, p, c = x.shape
    out = torch.empty((2, n, groups), dtype=torch.float64, device="cuda")
    for i in range(n):
        v = x[i].double().view(p, groups, c // groups)
        mean = v.mean((0, 2))
        out[0, i] = mean
        out[1, i] = 1 / ((v - mean[:, None]).square_().mean((0, 2)) + EPS).sqrt()
    return out


def _check_stats64(x, groups, stats):
    n, p, c = x.shape
    want = _stats64(x, groups)
    mag = torch.stack([x[i].abs().view(p, groups, -1).mean((0, 2), dtype=torch.float64) for i in range(n)])
    off = (stats.double() - want).abs()
    assert (off[0] <= K * mag).all(), ("mean", float((off[0] / mag).max()))
    assert (off[1] <= want[1] * (K + (K * mag * want[1]) ** 2)).all(), ("rstd", float((off[1] / want[1]).max()))
    return want


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("offset", [10.0, 1000.0])
@pytest.mark.parametrize("shape", [(224, 512, 1032, 8), (256, 4096, 1024, 32), (160, 4096, 264, 1), (1, 444 * 256 * 512, 1, 1)], ids=str)
def test_variance_where_a_thread_has_many_values(prec_name, offset, shape):
    """Hundreds of values a thread, the first of them 0 as at the border of a padded map, the rest far from 0.  What a thread's
    sums cancel must not grow with their number: the tolerance is that of the small cases."""
    _, ew = _ops(prec_name)
    n, p, c, groups = shape
    x = torch.empty((n, p, c), dtype=ew.dtype, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(11)
    for i in range(n):
        x[i] = torch.randn((p, c), generator=g, device="cuda") + offset
    rows = 256 // -(-c // 8)                         # of threads: the first pixels of an image, or of a CTA's share of it
    x.view(-1, 512 * 256 if c == 1 else p, c)[:, :rows] = 0
    gamma, beta = (_f32(a) for a in _params(c, 161))
    y, stats, _, _ = ew.gn_forward(x, groups, gamma, beta, eps=EPS)
    want = _check_stats64(x, groups, stats)
    wide = lambda t: t.repeat_interleave(c // groups)  # noqa: E731
    for i in {0, n - 1}:
        m, r, v = wide(want[0, i]), wide(want[1, i]), x[i].double()
        z = (v - m) * r * gamma + beta
        size = (v.abs() + m.abs()) * r * gamma.abs() + beta.abs()
        assert ((y[i].double() - z).abs() <= _half_step(ew.dtype) * z.abs() + 1.1 * K * size).all()


@pytest.mark.parametrize("offset", [1367.9, 535.4, 1501.1])
def test_variance_where_a_row_of_threads_differs(offset):
    """Maps of 256 pixels a row whose first column is blank: one of a CTA's 256 rows of threads has nothing but that column."""
    _, ew = _ops("fp32")
    for n, c, groups in ((1, 8, 1), (2, 16, 2)):
        x = torch.full((n, 65536, c), offset, device="cuda")
        x.view(n, 256, 256, c)[:, :, 0] = 0
        one, zero = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
        _check_stats64(x, groups, ew.gn_forward(x, groups, one, zero, eps=EPS)[1])
    # a last share of 50 pixels for 85 rows of threads
    x = torch.full((1, 150772, 24), offset, device="cuda")
    x[:, ::85] = 0
    _check_stats64(x, 3, ew.gn_forward(x, 3, torch.ones(24, device="cuda"), torch.zeros(24, device="cuda"), eps=EPS)[1])


# (N, pixels, C, groups) of every form: teams (one pixel, columns in one group and cut, slices), clusters, streamed with the rows of sums
# merged and combined, tiles of columns
FORMS = [(700, 1, 64, 4), (4096, 4, 30, 6), (500, 49, 40, 8), (500, 3, 4096, 32), (2, 1024, 160, 32), (128, 256, 48, 3), (130, 1024, 96, 32),
         (1, 16384, 64, 8), (2, 9001, 160, 32), (1, 20011, 30, 1), (1, 3, 2056, 8), (2, 40, 4104, 27), (30, 40, 4104, 513)]


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("shape", FORMS, ids=str)
def test_groups_without_spread(prec_name, shape):
    """Every value of a group the same: x - mean is 0 and y = act(beta), rounded once, whatever the value and gamma are."""
    _, ew = _ops(prec_name)
    n, p, c, groups = shape
    r = np.random.default_rng(171)
    level = _f32(r.choice([100.0, 3.3, -0.7, 4096.0, 1e4, -777.77, 0.0, 1e-3], (n, 1, groups))).to(ew.dtype)
    x = level.repeat_interleave(c // groups, -1).expand(n, p, c).contiguous()
    gamma = _f32(r.choice([1.0, 0.9, 1.13, -2.0], c))
    beta = _f32(r.choice([0.0, 0.25, -0.125, 1e-3], c))
    for act in ("none", "relu"):
        y, stats, bits, _ = ew.gn_forward(x, groups, gamma, beta, act=act, eps=EPS, gate=act == "relu")
        assert torch.equal(stats[0], level[:, 0].float()), "mean"
        assert ((stats[1].double() * EPS ** 0.5 - 1).abs() <= K).all(), "rstd"
        want = (beta if act == "none" else beta.clamp(min=0)).to(ew.dtype).expand(n, p, c)
        assert torch.equal(y, want), float((y.double() - want.double()).abs().max())
    bits = np.unpackbits(bits.cpu().numpy(), axis=-1, bitorder="little")[..., :c]
    assert (bits == (beta > 0).cpu().numpy()).all()


def test_silu_of_16_bit_tensors_far_from_zero():
    """As test_silu_over_its_range, to the ends: sigmoids down to the smallest normal number (a smaller one may be 0, which costs
    2^-126 (1 + |z|)), nothing beyond, infinities as a division has them.  A sigmoid of z < 0 is a product more, u, than there."""
    _, ew = _ops("bf16")
    c = 4096
    z = np.linspace(-120, 120, c).astype(np.float32)
    zz = z.astype(np.float64)
    x = torch.zeros(1, 1, c, device="cuda", dtype=ew.dtype)
    zero = torch.zeros(c, device="cuda")
    u = 2.0 ** -24
    s = 1 / (1 + np.exp(-zz))
    d = (2 * np.abs(zz) + 10) * u
    lost = 2.0 ** -126 * (1 + np.abs(zz))
    y, stats, _, _ = ew.gn_forward(x, 4, zero, _f32(z), act="silu")
    _near(y.reshape(c), zz * s, np.abs(zz * s) * (_half_step(ew.dtype) * (1 + 2 * d) + d + u) + lost, "y")
    _, _, db = ew.gn_backward(torch.ones_like(x), x, stats, 4, zero, _f32(z), act="silu")
    slope = s * (1 + zz * (1 - s))
    inner = np.abs(zz) * (d * s + 2 * u * (1 - s) + u) + u
    _near(db, slope, s * inner * (1 + 2 * d) + np.abs(slope) * (d + u) + lost, "dbeta")
    inf, nan = float("inf"), float("nan")
    ends = _f32([-1e4, -3e38, -inf, 1.0, nan, -1.0, inf, 3e38, -1e13, nan, -inf, -inf, 2.0, -60.0, -60.0, 60.0])
    x = torch.zeros(1, 1, 16, device="cuda", dtype=ew.dtype)
    y, stats, _, _ = ew.gn_forward(x, 4, zero[:16], ends, act="silu")
    got, want = y.reshape(16).double().cpu(), (ends.double() / (1 + (-ends.double()).exp())).cpu()
    assert torch.equal(got.isnan(), want.isnan()) and got[6] == inf
    fine = want.isfinite()
    assert ((got - want).abs()[fine] <= want.abs()[fine] * (2.0 ** -8 + 2.0 ** -15) + 1e-33).all(), (got, want)
    _, _, db = ew.gn_backward(torch.ones_like(x), x, stats, 4, zero[:16], ends, act="silu")
    s = torch.sigmoid(ends.double()).cpu()
    want = s * (1 + ends.double().cpu() * (1 - s))
    assert torch.equal(db.double().cpu().isnan(), want.isnan())
    fine = want.isfinite()
    assert ((db.double().cpu() - want).abs()[fine] <= want.abs()[fine] * 2.0 ** -15 + 1e-33).all(), (db, want)


@pytest.mark.parametrize("prec_name, shape, value", [("fp32", (1, 296 * 256 * 4096, 1, 1), 0.5108032), ("fp32", (150, 4096, 1032, 8), 0.5108032),
                                                      ("bf16", (150, 4096, 1032, 8), 0.51171875)], ids=str)
def test_gradients_where_a_thread_has_many_values(prec_name, shape, value):
    """Thousands of gradients a thread, all of them the same, as the mean of a map hands them down: no sum may drift with their
    number."""
    _, ew = _ops(prec_name)
    n, p, c, groups = shape
    x = torch.empty((n, p, c), dtype=ew.dtype, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(13)
    for i in range(n):
        x[i] = torch.randn((p, c), generator=g, device="cuda") * 1.3 + 0.4
    dy = torch.full_like(x, value)
    one = torch.ones(c, device="cuda")
    _, stats, _, _ = ew.gn_forward(x, groups, one, torch.zeros_like(one), eps=EPS)
    dx, dgamma, dbeta = ew.gn_backward(dy, x, stats, groups, one)
    v, wide = float(dy.view(-1)[0]), lambda t: t.double().repeat_interleave(c // groups)
    total = v * n * p
    assert ((dbeta.double() - total).abs() <= 2 * K * total).all(), float((dbeta.double() / total - 1).abs().max())
    A, mag = torch.zeros(c, dtype=torch.float64, device="cuda"), torch.zeros(c, dtype=torch.float64, device="cuda")
    for i in range(n):
        m, r = wide(stats[0, i]), wide(stats[1, i])
        A += v * ((x[i].double() - m) * r).sum(0)
        mag += v * (r * (x[i].double().abs() + m.abs())).sum(0)
    assert ((dgamma.double() - A).abs() <= 2 * K * mag).all()
    m, r, x0 = wide(stats[0, 0]), wide(stats[1, 0]), x[0].double()
    by = lambda t: wide(t.view(p, groups, c // groups).mean((0, 2)))  # noqa: E731
    xhat = (x0 - m) * r
    size = (x0.abs() + m.abs()) * r
    want = r * (v - v - xhat * by(v * xhat))
    assert ((dx[0].double() - want).abs() <= _half_step(ew.dtype) * want.abs() + 2 * K * r * (2 * v + size * by(v * size))).all()


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("act, gate, held, by", [("none", False, True, 0), ("relu", False, False, 0), ("relu", True, False, 0), ("relu", True, True, 0), ("silu", False, False, 0),
                                                 ("silu", False, True, 0), ("relu", True, True, 4), ("silu", False, False, 2), ("relu", False, False, 1)])
def test_gradients_of_long_threads_in_every_form(prec_name, act, gate, held, by):
    """More vectors a thread than a chain of sums has, against float64 on the GPU."""
    _, ew = _ops(prec_name)
    n, p, c, groups = 2, 148 * 90 + 5, 1032, 8
    buf = torch.empty(n * p * c + by, dtype=ew.dtype, device="cuda")
    x = buf[by:].view(n, p, c)
    x.copy_(torch.randn((n, p, c), generator=torch.Generator(device="cuda").manual_seed(23), device="cuda") * 1.3 + 0.4)
    dy = torch.randn((n, p, c), generator=torch.Generator(device="cuda").manual_seed(24), device="cuda").mul_(0.2).add_(0.5108032).to(ew.dtype)
    gamma, beta = (_f32(a) for a in _params(c, 231))
    y, stats, bits, kept = ew.gn_forward(x, groups, gamma, beta, act=act, gate=gate, checkpoint=held)
    dx, dgamma, dbeta = ew.gn_backward(dy, kept if held else x, stats, groups, gamma, beta, act=act, gate=bits, mask=y if act == "relu" and not gate else None)
    xo = (ew.ckpt_decode(kept) if held else x).double()
    for i in range(n):
        m, r = (stats[k, i].double().repeat_interleave(c // groups) for k in range(2))
        xhat, size = (xo[i] - m) * r, (xo[i].abs() + m.abs()) * r
        dz = dy[i].double()
        adz = dz.abs()
        if act == "relu":
            dz = dz * (y[i] > 0)
            adz = dz.abs()
        elif act == "silu":
            z = gamma * xhat + beta
            s = torch.sigmoid(z)
            dz, adz = dz * s * (1 + z * (1 - s)), (dz * s * (1 + z * (1 - s))).abs() + 0.5 * adz * (size * gamma.abs() + beta.abs())
        total = (dz * xhat).sum(0), dz.sum(0), (adz * size).sum(0), adz.sum(0)
        A, B, ma, mb = total if i == 0 else (s + t for s, t in zip((A, B, ma, mb), total))
        mean = lambda t: t.view(p, groups, -1).mean((0, 2)).repeat_interleave(c // groups)  # noqa: E731
        h = dz * gamma
        want = r * (h - mean(h) - xhat * mean(h * xhat))
        h = adz * gamma.abs()
        assert ((dx[i].double() - want).abs() <= _half_step(ew.dtype) * want.abs() + 2 * K * r * (h + mean(h) + size * mean(h * size))).all()
    assert ((dgamma.double() - A).abs() <= 2 * K * ma).all() and ((dbeta.double() - B).abs() <= 2 * K * mb).all()


def test_buffers_written_anew_for_every_call():
    """Codes, scales, bits and scratch in the same buffers call after call, with nothing between the calls: each backward pass
    reads what the forward pass before it left."""
    B, ew = _ops("bf16")
    lib, prec, st = ew.lib, ew.precision, torch.cuda.current_stream().cuda_stream
    for n, p, c, groups in ((8, 1024, 160, 32), (2, 12000, 96, 8), (2000, 4, 64, 4)):
        s, need, back = B.fdg_gn_shape(n, p, c, groups), C.c_size_t(), C.c_size_t()
        assert lib.fdg_gn_scratch_bytes(prec, C.byref(s), 0, C.byref(need)) == 0
        assert lib.fdg_gn_scratch_bytes(prec, C.byref(s), 1, C.byref(back)) == 0
        gamma, beta = (_f32(a) for a in _params(c, 201))
        ins = [(_mk((n, p, c), 202 + i, ew.dtype)[0], _mk((n, p, c), 212 + i, ew.dtype)[0]) for i in range(4)]
        y = torch.empty_like(ins[0][0])
        stats = torch.empty((2, n, groups), device="cuda")
        bits, codes, scales, scratch = (torch.empty(k, dtype=torch.uint8, device="cuda") for k in
                                        (n * p * (c // 8), n * p * c, n * p * -(-c // 32), max(need.value, back.value, 1)))
        got = []
        torch.cuda.synchronize()
        for k in range(12):
            x, dy = ins[k % 4]
            dx, dg, db = torch.empty_like(x), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
            assert lib.fdg_gn_forward(prec, C.byref(s), x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), None, B.FDG_ACT_RELU, EPS, y.data_ptr(),
                                      stats.data_ptr(), bits.data_ptr(), codes.data_ptr(), scales.data_ptr(), scratch.data_ptr(), need.value, st) == 0
            assert lib.fdg_gn_backward(prec, C.byref(s), dy.data_ptr(), None, codes.data_ptr(), scales.data_ptr(), stats.data_ptr(), gamma.data_ptr(), None,
                                       B.FDG_ACT_RELU, None, bits.data_ptr(), None, dx.data_ptr(), dg.data_ptr(), db.data_ptr(), scratch.data_ptr(),
                                       back.value, st) == 0
            got.append((dx, dg, db))
        torch.cuda.synchronize()
        for k, (x, dy) in enumerate(ins):
            _, stats1, bits1, held1 = ew.gn_forward(x, groups, gamma, beta, act="relu", gate=True, checkpoint=True)
            torch.cuda.synchronize()
            want = ew.gn_backward(dy, held1, stats1, groups, gamma, act="relu", gate=bits1)
            for j in range(k, 12, 4):
                assert all(torch.equal(a, b) for a, b in zip(got[j], want)), (k, j)


def test_more_groups_and_totals_than_a_grid_has_ctas():
    """The statistics of many groups and the totals of many images, each formed by a launch of its own of bounded size."""
    _, ew = _ops("bf16")
    for shape in ((12, 40, 4104, 1026), (16, 70, 4104, 4104), (3, 300, 2064, 2064)):
        n, p, c, groups = shape
        x, xo, y, stats, bits, _ = _check_forward(ew, shape, "relu", False, seed=220, gate=True)
        _check_backward(ew, shape, "relu", 220, xo, x, stats, y, bits, True, False)


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("shape", [(8, 256, 8, 4), (2, 1024, 160, 32), (3, 65, 33, 11), (1, 16384, 64, 8), (2, 9001, 160, 32), (1, 20011, 30, 1),
                                   (2, 5, 4104, 27), (2000, 4, 64, 4), (1100, 25, 96, 4), (601, 21, 30, 6), (300, 1, 4096, 32)], ids=str)
def test_the_options_of_the_backward_pass_together(prec_name, shape):
    """The stored y and a gradient added to dx, with x and with its codes; x with bits, with and without the added gradient."""
    _, ew = _ops(prec_name)
    n, p, c, groups = shape
    x, xo, y, stats, bits, _ = _check_forward(ew, shape, "relu", True, seed=180, gate=True)
    held = ew.ckpt_encode(x)
    heldo = L.ckpt_decode(held[0].cpu().numpy().reshape(-1, c), held[1].cpu().numpy().reshape(n * p, -1)).reshape(n, p, c)
    for xo_, x_ in ((xo, x), (heldo, held)):
        for with_res in (False, True):
            a = _check_backward(ew, shape, "relu", 180, xo_, x_, stats, y, bits, with_res, False)
            b = _check_backward(ew, shape, "relu", 180, xo_, x_, stats, y, bits, with_res, True)
            assert all(torch.equal(s, t) for s, t in zip(a, b))          # the gate is the same, so is everything


@pytest.mark.parametrize("prec_name", PRECISIONS)
@pytest.mark.parametrize("by", [0, 1, 2, 4])
@pytest.mark.parametrize("shape", LARGE + [(1, 20000, 36, 4), (2, 12000, 96, 8), (1, 70001, 16, 2), (1, 50000, 8, 1), (2, 3000, 2112, 33)], ids=str)
def test_codes_of_streamed_calls_are_those_of_the_encoder(prec_name, shape, by):
    _, ew = _ops(prec_name)
    n, p, c, groups = shape
    buf = torch.empty(n * p * c + by, dtype=ew.dtype, device="cuda")
    x = buf[by:].view(n, p, c)
    x.copy_(torch.randn((n, p, c), generator=torch.Generator(device="cuda").manual_seed(19), device="cuda") * 2 + 0.5)
    x[0, 17, :3], x[-1, p - 1, c - 1] = 0.0, float("inf")
    want = ew.ckpt_encode(x)
    gamma, beta = (_f32(a) for a in _params(c, 191))
    for act, kw in (("relu", dict(gate=True)), ("none", dict(res=x)), ("silu", {})):
        held = ew.gn_forward(x, groups, gamma, beta, act=act, checkpoint=True, **kw)[3]
        assert torch.equal(held[0], want[0]) and torch.equal(held[1], want[1])


def test_sums_of_parameters_past_32_bits():
    """More than 2^31 values: dgamma and dbeta, against float64 sums image by image."""
    _, ew = _ops("bf16")
    n, p, c, groups = 17, 1 << 20, 128, 8
    x = torch.empty((n, p, c), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(6)
    for i in range(n):
        x[i] = torch.randn((p, c), generator=g, device="cuda")
    one = torch.ones(c, device="cuda")
    y, stats, _, _ = ew.gn_forward(x, groups, one, torch.zeros_like(one), act="relu")
    dx, dgamma, dbeta = ew.gn_backward(y, x, stats, groups, one, act="relu", mask=y)
    A, B, mag = (torch.zeros(c, dtype=torch.float64, device="cuda") for _ in range(3))
    for i in range(n):
        for first in range(0, p, 1 << 18):
            v, dz = x[i, first:first + (1 << 18)].double(), y[i, first:first + (1 << 18)].double()
            m, r = (stats[k, i].double().repeat_interleave(c // groups) for k in range(2))
            A += (dz * (v - m) * r).sum(0)
            B += dz.sum(0)
            mag += (dz * (v.abs() + m.abs()) * r).sum(0)
    assert ((dgamma.double() - A).abs() <= 2 * K * mag).all() and ((dbeta.double() - B).abs() <= 2 * K * B).all()
