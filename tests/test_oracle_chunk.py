"""Pins of the chunk oracle: nothing here compares it with itself."""
import numpy as np
import pytest
import torch

from oracle import chunk_oracle as CO
from oracle import fasa_oracle as O


def test_e4m3_values_are_torchs():
    want = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(CO.e4m3_values(), want)
    assert np.nanmax(CO.e4m3_values()) == CO.E4M3_LARGEST


def test_hand_worked_rows():
    x = np.zeros((4, 128))
    x[0, :6] = [127.0, 0.5, 1.5, -2.5, 3.49, -126.5]         # scale 1: ties go to even
    x[1, :4] = [-254.0, 1.0, 3.0, 5.0]                        # scale 2
    x[3, 9] = -1e-3
    c, s = CO.quantise(x, "int8")
    assert s.tolist() == [1.0, 2.0, 0.0, np.float32(1e-3 / 127)]
    assert CO.values(c, "int8")[0, :6].tolist() == [127, 0, 2, -2, 3, -126]
    assert CO.values(c, "int8")[1, :4].tolist() == [-127, 0, 2, 2] and not c[2].any() and CO.values(c, "int8")[3, 9] == -127
    x[0, :8] = [448.0, 17.0, 19.0, -21.0, 0.0009765625, 0.0029296875, 0.001, 432.0]   # steps of 2 from 16 on, of 2^-9 up to 2^-6
    c, s = CO.quantise(x[:1], "e4m3")
    assert s[0] == 1.0 and CO.values(c, "e4m3")[0, :8].tolist() == [448, 16, 20, -20, 0, 2 * 2.0 ** -9, 2.0 ** -9, 448]


def test_e4m3_rounding_is_torchs():
    y = np.random.default_rng(0).standard_normal((500, 128)) * 2.0 ** np.random.default_rng(1).integers(-9, 6, (500, 1))
    y = y.astype(np.float32).astype(np.float64).clip(-447, 447)
    y[:, 0] = 448.0                                             # scale 1
    c, s = CO.quantise(y, "e4m3")
    assert (s == 1).all()
    np.testing.assert_array_equal(CO.values(c, "e4m3"), torch.from_numpy(y).to(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("fmt,step", [("int8", 0.5 / 127), ("e4m3", 2.0 ** -4)])
def test_dequantised_rows_are_within_half_a_step(fmt, step):
    x = np.random.default_rng(2).standard_normal((200, 128))
    back = CO.dequantise(*CO.quantise(x, fmt), fmt)
    top = np.abs(x).max(-1, keepdims=True)
    bound = step * top if fmt == "int8" else np.maximum(step * np.abs(x), 2.0 ** -10 / 448 * top)
    assert (np.abs(back - x) <= bound * (1 + 1e-6)).all()


def test_rows_that_are_not_finite():
    x = np.ones((3, 128))
    x[0, 3], x[1, 4] = np.inf, np.nan
    c, s = CO.quantise(x, "int8")
    assert np.isnan(s[:2]).all() and s[2] == np.float32(1 / 127) and not c[:2].any()


def test_attention_is_torchs_and_one_token_is_dense():
    rng = np.random.default_rng(3)
    n, G, N = 9, 3, 30
    q, K, V = rng.standard_normal((n, G, 128)), rng.standard_normal((N, 128)), rng.standard_normal((N, 128))
    got, A, L = CO.chunk_attend(q, K, V)
    mask = torch.ones(n, N, dtype=torch.bool).tril(N - n)
    t = torch.from_numpy
    want = torch.nn.functional.scaled_dot_product_attention(t(q).transpose(0, 1), t(K).expand(G, N, 128), t(V).expand(G, N, 128), attn_mask=mask).transpose(0, 1)
    np.testing.assert_allclose(got, want.numpy(), rtol=1e-12, atol=1e-13)
    assert (np.abs(got) <= A + 1e-15).all() and (L > 0).all()
    one = CO.chunk_attend(q[-1:].astype(np.float32).astype(np.float64), K.astype(np.float32).astype(np.float64), V.astype(np.float32).astype(np.float64))[0]
    dense = O.dense_attend(q[-1:].astype(np.float32), K[None, None].astype(np.float32), V[None, None].astype(np.float32), N)
    np.testing.assert_allclose(one, dense, rtol=1e-12, atol=1e-13)
