"""Pins of the dense operators' plain implementations against things other than themselves: the generator's published test
vectors, library layers and autograd in fp64, central differences, and counts that the probability implies."""
import numpy as np
import pytest
import torch

from oracle import dense

ACTS = ["none", "relu", "gelu", "silu"]


def test_generator_known_answers():
    """The test vectors that its authors publish with the generator (philox4x32-10)."""
    assert [hex(w) for w in dense.philox(0, 0, 0, 1)[0]] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
    ones = 2 ** 64 - 1
    assert [hex(w) for w in dense.philox(ones, ones, ones, 1)[0]] == ["0x408f276d", "0x41c83b0e", "0xa20bc7c6", "0x6d5451fd"]


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9])
def test_share_of_dropped_elements(p):
    n = 1 << 18
    dropped = n - int(dense.keep((n,), p, 12, 34).sum())
    assert abs(dropped - n * p) <= 6 * np.sqrt(n * p * (1 - p))  # six standard deviations
    assert p == 0.0 or (dense.keep((n,), p, 12, 34) != dense.keep((n,), p, 12, 35)).any()


def _t(a):
    return torch.from_numpy(a).requires_grad_(True)


LIB = {"none": lambda z: z, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_linear_equals_library_autograd(name, p):
    g = np.random.default_rng(3)
    x, w, b, r, dout = g.normal(size=(13, 7)), g.normal(size=(5, 7)), g.normal(size=5), g.normal(size=(13, 5)), g.normal(size=(13, 5))
    rng = (77, -5)
    out, pre = dense.linear_fwd(x, w, b, r, name, p, rng)
    tx, tw, tb = _t(x), _t(w), _t(b)
    mask = torch.from_numpy(dense.keep((13, 5), p, *rng)) if p else torch.ones(13, 5, dtype=torch.bool)
    ref = torch.from_numpy(r) + LIB[name](torch.nn.functional.linear(tx, tw, tb)) * mask / (1 - float(np.float32(p)))
    assert np.allclose(out, ref.detach().numpy(), rtol=1e-12, atol=1e-12)
    ref.backward(torch.from_numpy(dout))
    got = dense.linear_bwd(x, w, dout, pre, name, p, rng)
    for key, t in (("dx", tx), ("dweight", tw), ("dbias", tb)):
        assert np.allclose(got[key], t.grad.numpy(), rtol=1e-11, atol=1e-11), key


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("B,N,C,G", [(3, 6, 8, 2), (2, 5, 6, 6), (4, 1, 10, 1)])
def test_norm_equals_library_autograd(name, B, N, C, G):
    g = np.random.default_rng(4)
    x, gamma, beta, dout = g.normal(size=(B, N, C)) + 0.5, g.normal(size=C), g.normal(size=C), g.normal(size=(B, N, C))
    out, mean, rstd = dense.norm_fwd(x, gamma, beta, G, 1e-5, name)
    tx, tg, tb = _t(x), _t(gamma), _t(beta)
    ref = LIB[name](torch.nn.functional.group_norm(tx.transpose(1, 2), G, tg, tb, 1e-5).transpose(1, 2))
    assert np.allclose(out, ref.detach().numpy(), rtol=1e-11, atol=1e-11)
    ref.backward(torch.from_numpy(dout))
    got = dense.norm_bwd(x, gamma, beta, mean, rstd, dout, G, name)
    for key, t in (("dx", tx), ("dgamma", tg), ("dbeta", tb)):
        assert np.allclose(got[key], t.grad.numpy(), rtol=1e-9, atol=1e-10), key


@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_gradients_are_differences(name):
    g = np.random.default_rng(5)
    x, w, b, dout = g.normal(size=(6, 4)), g.normal(size=(3, 4)), g.normal(size=3), g.normal(size=(6, 3))
    rng, p, h = (9, 1), 0.4, 1e-6

    def loss(x, w, b):
        return float((dense.linear_fwd(x, w, b, None, name, p, rng)[0] * dout).sum())

    got = dense.linear_bwd(x, w, dout, dense.linear_fwd(x, w, b)[1], name, p, rng)
    for key, arg in (("dx", 0), ("dweight", 1), ("dbias", 2)):
        args = [x, w, b]
        for i in np.ndindex(args[arg].shape):
            d = np.zeros_like(args[arg])
            d[i] = h
            up, down = list(args), list(args)
            up[arg], down[arg] = args[arg] + d, args[arg] - d
            assert abs((loss(*up) - loss(*down)) / (2 * h) - got[key][i]) < 1e-7, (key, i)
    xn, gamma, beta, dn = g.normal(size=(2, 3, 4)), g.normal(size=4), g.normal(size=4), g.normal(size=(2, 3, 4))

    def nloss(x, gamma, beta):
        return float((dense.norm_fwd(x, gamma, beta, 2, 1e-5, name)[0] * dn).sum())

    _, mean, rstd = dense.norm_fwd(xn, gamma, beta, 2, 1e-5, name)
    got = dense.norm_bwd(xn, gamma, beta, mean, rstd, dn, 2, name)
    for key, arg in (("dx", 0), ("dgamma", 1), ("dbeta", 2)):
        args = [xn, gamma, beta]
        for i in np.ndindex(args[arg].shape):
            d = np.zeros_like(args[arg])
            d[i] = h
            up, down = list(args), list(args)
            up[arg], down[arg] = args[arg] + d, args[arg] - d
            assert abs((nloss(*up) - nloss(*down)) / (2 * h) - got[key][i]) < 1e-6, (key, i)
