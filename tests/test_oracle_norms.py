"""The oracle of group norm and of tensors held in 8 bits (oracle/norms.py), pinned without the library: against torch's
float64 autograd, against central differences, and against the properties the format promises."""
import numpy as np
import pytest
import torch

from oracle import norms as L

EPS = 1e-5
SHAPES = [(2, 6, 8, 4), (3, 1, 6, 2), (1, 9, 5, 1), (2, 4, 5, 5), (2, 7, 30, 6)]


def _rand(shape, seed):
    return np.random.default_rng(seed).standard_normal(shape)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("n, p, c, groups", SHAPES)
def test_forward_and_gradients_match_autograd(n, p, c, groups, act):
    x, res, dy = _rand((n, p, c), 1) * 2 + 0.7, _rand((n, p, c), 2), _rand((n, p, c), 3)
    gamma, beta = 1 + 0.3 * _rand(c, 4), 0.2 * _rand(c, 5)
    y, z, stats = L.groupnorm_forward(x, groups, gamma, beta, EPS, act, res)
    t = [torch.tensor(a, requires_grad=True) for a in (x, gamma, beta, res)]
    zt = torch.nn.functional.group_norm(t[0].movedim(-1, 1), groups, t[1], t[2], EPS).movedim(1, -1) + t[3]
    yt = {"none": lambda v: v, "relu": torch.relu, "silu": torch.nn.functional.silu}[act](zt)
    np.testing.assert_allclose(y, yt.detach().numpy(), rtol=1e-10, atol=1e-10)
    yt.backward(torch.tensor(dy))
    dz = dy * L.activation_slope(z, act)
    dx, dgamma, dbeta = L.groupnorm_backward(dz, x, stats, groups, gamma)
    for got, want in ((dx, t[0]), (dgamma, t[1]), (dbeta, t[2]), (dz, t[3])):
        np.testing.assert_allclose(got, want.grad.numpy(), rtol=1e-8, atol=1e-9)


def test_gradient_matches_differences():
    n, p, c, groups, h = 2, 5, 6, 3, 1e-5
    x, dy = _rand((n, p, c), 6) + 0.4, _rand((n, p, c), 7)
    gamma, beta = 1 + 0.3 * _rand(c, 8), 0.2 * _rand(c, 9)

    def loss(x, gamma, beta):
        return (L.groupnorm_forward(x, groups, gamma, beta, EPS, "silu")[0] * dy).sum()

    _, z, stats = L.groupnorm_forward(x, groups, gamma, beta, EPS, "silu")
    grads = L.groupnorm_backward(dy * L.activation_slope(z, "silu"), x, stats, groups, gamma)
    for which, (arg, grad) in enumerate(zip((x, gamma, beta), grads)):
        for i in range(0, arg.size, 7 if arg.size > 20 else 1):
            lo, hi = arg.copy().reshape(-1), arg.copy().reshape(-1)
            lo[i] -= h
            hi[i] += h
            args = [[x, gamma, beta], [x, gamma, beta]]
            args[0][which], args[1][which] = lo.reshape(arg.shape), hi.reshape(arg.shape)
            d = (loss(*args[1]) - loss(*args[0])) / (2 * h)
            # second order of the difference ~ h^2 times a third derivative of order 10, and 1e-16 / h of rounding
            assert abs(d - grad.reshape(-1)[i]) <= 1e-7, (which, i)


def test_held_values_are_the_nearest_of_the_smallest_steps():
    g = np.random.default_rng(10)
    x = g.standard_normal((40, 70)) * 10.0 ** g.integers(-30, 30, (40, 1))
    x[3] = 0.0
    codes, scales = L.ckpt_encode(x)
    back = L.ckpt_decode(codes, scales)
    for b in range(3):
        cols = slice(32 * b, min(32 * b + 32, 70))
        step = np.ldexp(1.0, scales[:, b].astype(int) - 127)
        top = np.abs(x[:, cols]).max(1)
        assert (np.abs(back[:, cols] - x[:, cols]).max(1) <= step / 2).all()
        assert (np.rint(top / step) <= 127).all()
        smaller = (np.rint(top / (step / 2)) > 127) | (scales[:, b] == 1)
        assert smaller.all()


def test_held_borders():
    x = np.zeros((6, 3))
    x[0] = 127.5, 1.0, 0.5          # 127.5 steps of 1 round to 128: the step is 2, and 1 = half a step goes to even
    x[1] = 127.49, 0.5, 1.5         # steps of 1, ties to even
    x[2] = np.nan, 1.0, 2.0
    x[3] = np.inf, 1.0, 2.0
    x[4] = 3.3895313892515355e38, 0.0, -3.3895313892515355e38        # bf16's largest magnitude stays finite
    x[5] = 2.0 ** -149, 2.0 ** -126, -2.0 ** -127
    codes, scales = L.ckpt_encode(x)
    back = L.ckpt_decode(codes, scales)
    assert scales[0, 0] == 128 and back[0].tolist() == [128.0, 0.0, 0.0]
    assert scales[1, 0] == 127 and back[1].tolist() == [127.0, 0.0, 2.0]
    assert scales[2, 0] == scales[3, 0] == 255 and np.isnan(back[2]).all() and np.isnan(back[3]).all() and not codes[2:4].any()
    assert scales[4, 0] == 248 and np.isfinite(back[4]).all() and back[4, 0] == 127 * 2.0 ** 121
    assert scales[5, 0] == 1 and back[5].tolist() == [0.0, 2.0 ** -126, 0.0]
    # every value held is a bf16 number
    assert (torch.tensor(back[[0, 1, 4, 5]]).bfloat16().double().numpy() == back[[0, 1, 4, 5]]).all()
