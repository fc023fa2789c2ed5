"""What the operators around normalisation and activation checkpoints are measured on: group norm with an activation on
channels-last tensors (forward and backward) and tensors held in 8 bits, through `paper_1906_09108_b200.binding.EwOps`.

A case is one call of a training program on one layer (`op`):

  gn_forward    y = act(group norm of x [+ res]) and the statistics; with `ckpt` also x held in 8 bits, read back here as the
                values it stands for; with `gate` also the bits of [y > 0], which y itself shows
  gn_backward   dx, dgamma, dbeta from dy, the saved statistics and x, or (`ckpt`) x as it was held in 8 bits; ReLU's gate
                from the stored y, or from its bits (`gate`); `res`: a gradient added to dx
  ckpt          a tensor put into 8 bits and read back

8 bits: blocks of 32 consecutive channels of a pixel (the last block of a pixel may be shorter) share a scale 2^e, with e the
smallest integer >= -126 for which the largest magnitude rounds to at most 127 steps of 2^e; a value is held as the nearest
integer (ties to even) of such steps.

x has a mean and a spread of its own in every channel, as a convolution's output has; gradients are small.  Nothing is
returned for `gate`: whether a value within 32-bit rounding of zero is above it is no number that two ways of adding agree on.
"""
import math

import torch

own = False

BLOCK = 32


def _case(name, op, n, h, w, c, groups=0, dtype="bf16", act="none", res=False, gate=False, ckpt=False):
    d = dict(op=op, n=n, h=h, w=w, c=c, groups=groups, dtype=dtype, act=act, res=res, gate=gate, ckpt=ckpt)
    if name:
        d["name"] = name
    return d


def listed():
    return [
        # the smallest network there is a configuration for, its first stage: what a call costs when the kernel costs nothing
        _case("forward_tiny", "gn_forward", 8, 16, 16, 8, 4, act="relu"),
        # first stage of the deep narrow networks, with the shortcut added, as a post-activation block ends
        _case("forward_resnet110_stage1", "gn_forward", 128, 32, 32, 16, 4, act="relu", res=True),
        # first stage of the wide network: groups of five channels, the input kept in 8 bits and the gate in bits
        _case("forward_wrn_stage1_ckpt", "gn_forward", 128, 32, 32, 160, 32, act="relu", gate=True, ckpt=True),
        # exact mode on a batch, a map and a group that fill no tile
        _case("forward_fp32_ragged", "gn_forward", 37, 28, 28, 30, 6, dtype="fp32", act="silu"),
        # few images with many pixels: what one image has does not fit a cluster of SMs
        _case("forward_maps_256", "gn_forward", 8, 256, 256, 128, 32, act="silu"),
        # last stage of the wide network, its small maps, one group per image
        _case("backward_wrn_stage3", "gn_backward", 128, 8, 8, 640, 1, act="relu"),
        # the backward pass of forward_wrn_stage1_ckpt: x in 8 bits, the gate in bits, a shortcut's gradient added
        _case("backward_wrn_stage1_ckpt", "gn_backward", 128, 32, 32, 160, 32, act="relu", res=True, gate=True, ckpt=True),
        # exact mode, odd sizes
        _case("backward_fp32_ragged", "gn_backward", 37, 28, 28, 30, 6, dtype="fp32", act="silu"),
        # few images with many pixels, x in 8 bits
        _case("backward_maps_256_ckpt", "gn_backward", 8, 256, 256, 128, 32, act="silu", ckpt=True),
        # the smallest network's first stage
        _case("ckpt_tiny", "ckpt", 8, 16, 16, 8),
        # the widest tensor of the wide network
        _case("ckpt_wrn_stage1", "ckpt", 128, 32, 32, 160),
        # exact mode, channels that fill no block
        _case("ckpt_fp32_ragged", "ckpt", 97, 28, 28, 30, dtype="fp32"),
    ]


_MOST = 8 * 256 * 256 * 128          # elements of the largest listed case


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Layers between the listed ones: batch, map, channels, groups, storage type and options."""
    op = rng.choice(("gn_forward", "gn_forward", "gn_backward", "gn_backward", "ckpt"))
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    most = _MOST // 4 if dtype == "fp32" else _MOST // 2
    h = _log_int(rng, 1, 256)
    w = h if rng.random() < 0.7 else _log_int(rng, 1, 256)
    unit = rng.choice((1, 2, 8, 8, 16, 32))
    c = min(unit * _log_int(rng, 1, max(1, 1024 // unit)), 1024)
    c = max(1, min(c, most // (h * w)))
    n = min(_log_int(rng, 1, 256), max(1, most // (h * w * c)))
    if op == "ckpt":
        return _case(None, op, n, h, w, c, 0, dtype)
    # groups of a handful of values are left to the forward pass: the mean and the spread take two degrees of freedom of a
    # group's gradient away, so a group of two has none but what eps leaves
    least = 32 if op == "gn_backward" else 1
    groups = rng.choice([g for g in range(1, c + 1) if c % g == 0 and h * w * c // g >= least] or [1])
    if h * w * c // groups < least:
        op = "gn_forward"
    act = rng.choice(("none", "relu", "relu", "silu"))
    return _case(None, op, n, h, w, c, groups, dtype, act, res=rng.random() < 0.3 and (act != "silu" or op == "gn_backward"),
                 gate=act == "relu" and rng.random() < 0.5, ckpt=rng.random() < 0.4)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ---- 8 bits, plainly ------------------------------------------------------------------------------------------------

def _encode(x):
    """(codes int8 like x, exponents + 127 uint8 [..., blocks]) of a tensor of finite values."""
    c = x.shape[-1]
    blocks = -(-c // BLOCK)
    v = torch.nn.functional.pad(x.float(), (0, blocks * BLOCK - c)).reshape(*x.shape[:-1], blocks, BLOCK)
    bits = v.abs().amax(-1).view(torch.int32)
    # exponent of the largest magnitude, one more where its mantissa is 255/128 or above (127.5 steps and more); 6 lower:
    # that is the exponent of a step
    k = (((bits + 0x10000) >> 23).clamp(max=254) - 6).clamp(min=1)
    steps = v * ((254 - k) << 23).view(torch.float32).unsqueeze(-1)        # a power of two: exact
    codes = steps.round().clamp(-127, 127).to(torch.int8).reshape(*x.shape[:-1], blocks * BLOCK)[..., :c].contiguous()
    return codes, k.to(torch.uint8)


def _decode(codes, scales):
    """The values that codes and scales stand for, in 32 bits."""
    step = (scales.int() << 23).view(torch.float32).repeat_interleave(BLOCK, -1)[..., :codes.shape[-1]]
    return codes.float() * step


def _pack(mask):
    """Bits of a truth tensor [..., c], eight channels a byte, the lowest channel lowest."""
    c = mask.shape[-1]
    m = torch.nn.functional.pad(mask.to(torch.uint8), (0, -c % 8)).reshape(*mask.shape[:-1], -1, 8)
    return (m << torch.arange(8, device=mask.device, dtype=torch.uint8)).sum(-1, dtype=torch.int32).to(torch.uint8)


def _unpack(bits, c):
    m = (bits.unsqueeze(-1) >> torch.arange(8, device=bits.device, dtype=torch.uint8)) & 1
    return m.reshape(*bits.shape[:-1], -1)[..., :c].bool()


# ---- inputs ---------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, h, w, c, groups = case["n"], case["h"], case["w"], case["c"], case["groups"]
    dt = _dtype(case)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    spread = 0.5 + torch.rand(c, generator=gen, device="cuda")
    x = (normal(n, h, w, c) * spread + 0.5 * normal(c)).to(dt)
    s = dict(case=case, x=x, eps=1e-5)
    if case["op"] == "ckpt":
        return s
    s.update(gamma=1 + 0.2 * normal(c), beta=0.1 * normal(c))
    s["res"] = normal(n, h, w, c).to(dt) if case["res"] else None
    if case["op"] == "gn_forward":
        return s
    s["dy"] = (1e-3 * normal(n, h, w, c)).to(dt)
    if s["res"] is not None:
        s["res"] = (1e-3 * s["res"]).to(dt)
    v = x.double().reshape(n, h * w, groups, c // groups)
    mean = v.mean((1, 3))
    rstd = ((v - mean[:, None, :, None]).square().mean((1, 3)) + s["eps"]).rsqrt()
    s["stats"] = torch.stack((mean, rstd)).float().contiguous()
    if case["act"] == "relu":
        z = ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(x.shape) * s["gamma"] + s["beta"]
        y = z.clamp(min=0).to(dt)
        s["mask"], s["gate"] = (None, _pack(y > 0)) if case["gate"] else (y, None)
    else:
        s["mask"] = s["gate"] = None
    if case["ckpt"]:
        s["held"] = _encode(x)
        s["x"] = None
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _grouped(t, case):
    return t.reshape(case["n"], case["h"] * case["w"], case["groups"], case["c"] // case["groups"])


def _plain_forward(s):
    case, dt = s["case"], s["x"].dtype
    x = _grouped(s["x"].float(), case)
    mean = x.mean((1, 3))
    d = x - mean[:, None, :, None]
    rstd = 1 / (d.square().mean((1, 3)) + s["eps"]).sqrt()
    z = (d * rstd[:, None, :, None]).reshape(s["x"].shape) * s["gamma"] + s["beta"]
    if s["res"] is not None:
        z = z + s["res"].float()
    if case["act"] == "relu":
        z = z.clamp(min=0)
    elif case["act"] == "silu":
        z = z / (1 + (-z).exp())
    out = dict(y=z.to(dt), stats=torch.stack((mean, rstd)))
    if case["gate"]:
        s["bits"] = _pack(out["y"] > 0)
    if case["ckpt"]:
        out["held"] = _decode(*_encode(s["x"])).to(dt)
    return out


def _plain_backward(s):
    case, dt = s["case"], s["dy"].dtype
    x = _decode(*s["held"]) if case["ckpt"] else s["x"].float()
    mean, rstd = s["stats"][0][:, None, :, None], s["stats"][1][:, None, :, None]
    xhat = (_grouped(x, case) - mean) * rstd
    flat = xhat.reshape(x.shape)
    dz = s["dy"].float()
    if case["act"] == "relu":
        dz = dz * (_unpack(s["gate"], case["c"]) if case["gate"] else s["mask"] > 0)
    elif case["act"] == "silu":
        z = flat * s["gamma"] + s["beta"]
        sig = 1 / (1 + (-z).exp())
        dz = dz * (sig * (1 + z * (1 - sig)))
    dgamma, dbeta = (dz * flat).sum((0, 1, 2)), dz.sum((0, 1, 2))
    g = _grouped(dz * s["gamma"], case)
    dx = rstd * (g - g.mean((1, 3), keepdim=True) - xhat * (g * xhat).mean((1, 3), keepdim=True))
    dx = dx.reshape(x.shape)
    if s["res"] is not None:
        dx = dx + s["res"].float()
    return dict(dx=dx.to(dt), dgamma=dgamma, dbeta=dbeta)


# ---- the framework's calls --------------------------------------------------------------------------------------------

_ops = {}


def _ew(case):
    """The framework's operators of a storage type, as a program keeps them."""
    if case["dtype"] not in _ops:
        from paper_1906_09108_b200 import binding as B
        _ops[case["dtype"]] = B.EwOps(B.FDG_BF16_TC if case["dtype"] == "bf16" else B.FDG_FP32_CUDACORE)
    return _ops[case["dtype"]]


def run(s):
    case = s["case"]
    if own:
        ew = _ew(case)
        if case["op"] == "ckpt":
            return ew.ckpt_decode(ew.ckpt_encode(s["x"]))
        if case["op"] == "gn_forward":
            y, stats, _, held = ew.gn_forward(s["x"], case["groups"], s["gamma"], s["beta"], act=case["act"], res=s["res"],
                                              eps=s["eps"], gate=case["gate"], checkpoint=case["ckpt"])
            return dict(y=y, stats=stats) if held is None else dict(y=y, stats=stats, held=ew.ckpt_decode(held))
        dx, dgamma, dbeta = ew.gn_backward(s["dy"], s["held"] if case["ckpt"] else s["x"], s["stats"], case["groups"],
                                           s["gamma"], s["beta"], act=case["act"], mask=s["mask"], gate=s["gate"], res=s["res"])
        return dict(dx=dx, dgamma=dgamma, dbeta=dbeta)
    if case["op"] == "ckpt":
        return _decode(*_encode(s["x"])).to(s["x"].dtype)
    return _plain_forward(s) if case["op"] == "gn_forward" else _plain_backward(s)


def work(case):
    n, c = case["n"], case["c"]
    pixels = case["h"] * case["w"]
    elems = n * pixels * c
    b = 2 if case["dtype"] == "bf16" else 4
    held = elems + n * pixels * -(-c // BLOCK)
    bits = n * pixels * -(-c // 8)
    if case["op"] == "ckpt":
        return dict(bytes=2 * elems * b + 2 * held, flops=4 * elems)
    stats = 8 * n * case["groups"] + 8 * c
    if case["op"] == "gn_forward":
        moved = 2 * elems * b + case["res"] * elems * b + case["gate"] * bits + case["ckpt"] * (2 * held + elems * b)
        return dict(bytes=moved + stats, flops=(9 + 6 * (case["act"] == "silu")) * elems)
    mask = 0 if case["act"] != "relu" else bits if case["gate"] else elems * b
    moved = 2 * elems * b + (held if case["ckpt"] else elems * b) + mask + case["res"] * elems * b
    return dict(bytes=moved + stats + 8 * c, flops=(14 + 10 * (case["act"] == "silu")) * elems)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------

def _two_to(e):
    """2^e in 64 bits for integers e, by its bits: pow() is off in the last place, which would move ties."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _held_exactly(x):
    """What a tensor held in 8 bits stands for: block by block, the smallest power of two in whose steps the largest
    magnitude rounds to at most 127."""
    c = x.shape[-1]
    v = x.double().reshape(-1, c)
    out = torch.empty_like(v)
    for first in range(0, c, BLOCK):
        part = v[:, first:first + BLOCK]
        top = part.abs().amax(1, keepdim=True)
        e = torch.frexp(top).exponent - 7
        e = torch.where(torch.round(top * _two_to(-e)) > 127, e + 1, e).clamp(min=-126)
        out[:, first:first + BLOCK] = torch.round(part * _two_to(-e)) * _two_to(e)
    return out.reshape(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "ckpt":
        return _held_exactly(s["x"])
    n, c, groups = case["n"], case["c"], case["groups"]

    def rows(t):
        """[image][group][pixel and channel within the group]."""
        t = t.double().reshape(n, -1, groups, c // groups)
        return t.permute(0, 2, 1, 3).reshape(n, groups, -1)

    def back(t, like):
        return t.reshape(n, groups, -1, c // groups).permute(0, 2, 1, 3).reshape(like.shape)

    gamma, beta = s["gamma"].double(), s["beta"].double()
    if case["op"] == "gn_forward":
        x = rows(s["x"])
        var, mean = torch.var_mean(x, -1, unbiased=False)
        rstd = torch.pow(var + s["eps"], -0.5)
        z = torch.addcmul(beta, back((x - mean[..., None]) * rstd[..., None], s["x"]), gamma)
        if s["res"] is not None:
            z += s["res"].double()
        y = torch.relu(z) if case["act"] == "relu" else z * torch.sigmoid(z) if case["act"] == "silu" else z
        out = dict(y=y, stats=torch.stack((mean, rstd)))
        if case["ckpt"]:
            out["held"] = _held_exactly(s["x"])
        return out
    dy = s["dy"].double()
    if case["ckpt"]:
        codes, k = s["held"]
        held = codes.double() * _two_to(k.long() - 127).repeat_interleave(BLOCK, -1)[..., :c]
    else:
        held = s["x"]
    mean, rstd = s["stats"].double().unbind(0)
    xhat = (rows(held) - mean[..., None]) * rstd[..., None]
    xflat = back(xhat, dy)
    if case["act"] == "relu":
        dz = torch.where(_unpack(s["gate"], c) if case["gate"] else s["mask"] > 0, dy, 0.0)
    elif case["act"] == "silu":
        z = torch.addcmul(beta, xflat, gamma)
        sig = torch.sigmoid(z)
        dz = dy * (sig + z * sig * torch.sigmoid(-z))
    else:
        dz = dy
    g = rows(dz * gamma)
    m = g.shape[-1]
    inner = torch.einsum("ngi,ngi->ng", g, xhat)
    dx = back(rstd[..., None] * (g - (g.sum(-1)[..., None] + xhat * inner[..., None]) / m), dy)
    if s["res"] is not None:
        dx = dx + s["res"].double()
    return dict(dx=dx, dgamma=torch.einsum("nhwc,nhwc->c", dz, xflat), dbeta=dz.sum((0, 1, 2)))
