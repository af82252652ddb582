"""The serving oracle on the CPU: its e4m3 numbers against torch's, paged
attention against the contiguous oracle and closed forms, placement of positions,
the activations against torch's."""
import numpy as np
import pytest

import oracle
from oracle import serving
from paper_2504_17577_amd import gen

torch = pytest.importorskip("torch")


def test_e4m3_codes_are_torch_s():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(serving.e4m3_values(), want)
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    x = x[~x.isnan()]
    mid = (want[:126] + want[1:127]) / 2          # ties
    x = torch.cat([x, torch.tensor(np.concatenate([mid, -mid]), dtype=torch.float32)])
    got = serving.e4m3_codes(x.numpy())
    ref = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(got, ref)
    assert np.isnan(serving.e4m3_values()[serving.e4m3_codes(np.array([np.nan]))]).all()


@pytest.mark.parametrize("Hq,Hkv,D,P", [(4, 2, 64, 16), (3, 1, 128, 32)])
def test_paged_attention_is_contiguous_attention(Hq, Hkv, D, P):
    B, n = 2, 50
    per = -(-n // P)
    q, k, v = gen.random_problem(B, Hq, Hkv, 1, n, D, seed=1)
    rng = np.random.default_rng(0)
    table = rng.permutation(B * per + 3)[:B * per].reshape(B, per)
    shape = (B * per + 3, Hkv, P, D)
    kc, vc = np.full(shape, np.nan), np.full(shape, np.nan)
    for b in range(B):
        for t in range(n):
            kc[table[b, t // P], :, t % P] = gen.f32_from_bf16(k[b, :, t])
            vc[table[b, t // P], :, t % P] = gen.f32_from_bf16(v[b, :, t])
    ro, rl = oracle.attn_fwd(q, k, v, False, 0.2)
    o, lse, tol, tol_lse = serving.attn_paged(gen.f32_from_bf16(q[:, :, 0]).astype(np.float64), kc, vc, table,
                                              [n] * B, 0.2)
    np.testing.assert_allclose(o, ro[:, :, 0], atol=1e-12)
    np.testing.assert_allclose(lse, rl[:, :, 0], atol=1e-12)
    # (0.2 * 132 * 2^-24 * 128 terms of at most 8 in the dot products, twice, for |V| up to 5)
    assert (tol > 0).all() and tol.max() < 2e-2 and tol_lse.max() < 2e-3


def test_attention_of_few_positions():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(3, 2, 64)), rng.normal(size=(4, 1, 16, 64)), rng.normal(size=(4, 1, 16, 64))
    table = np.array([[2, 0], [1, -1], [3, 9]])
    o, lse, _, _ = serving.attn_paged(q, k, v, table, [0, 1, 17], 1.0, np.array([0.5]), np.array([2.0]))
    assert (o[0] == 0).all() and (lse[0] == -np.inf).all()
    np.testing.assert_allclose(o[1], np.stack([2 * v[1, 0, 0]] * 2))
    np.testing.assert_allclose(lse[1], 0.5 * q[1] @ k[1, 0, 0])
    assert np.isnan(o[2]).all() and np.isnan(lse[2]).all()       # page 9 of 4


def test_places():
    table = np.array([[2, 0, -1], [1, 4, 3]])
    at = lambda seq, pos: serving.place(table, 4, 16, seq, pos)   # noqa: E731
    assert at(0, 0) == (2, 0) and at(0, 31) == (0, 15) and at(1, 47) == (3, 15)
    assert at(0, -1) is at(0, 48) is at(2, 0) is at(-1, 0) is at(0, 32) is at(1, 16) is None


@pytest.mark.parametrize("name", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_activations_are_torch_s(name):
    x = torch.linspace(-12, 12, 2001, dtype=torch.float64)
    f = torch.nn.functional
    want = {"none": lambda y: y, "relu": f.relu, "gelu": f.gelu, "silu": f.silu,
            "gelu_tanh": lambda y: f.gelu(y, approximate="tanh")}[name](x)
    np.testing.assert_allclose(serving.activated(x.numpy(), name), want.numpy(), atol=1e-14)
    slope = np.diff(want.numpy()) / 0.012
    assert np.abs(slope).max() <= 1.13
