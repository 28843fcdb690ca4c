"""The 8-bit cache's oracle: e4m3 by its bits, scales at their borders, layouts, attention against library routines."""
import numpy as np
import pytest

from oracle import kv8 as o8

torch = pytest.importorskip("torch")


def test_e4m3_is_torchs():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(o8.e4m3_decode(codes), want)
    x = np.random.default_rng(0).standard_normal(20000) * np.exp(np.random.default_rng(1).uniform(-8, 6, 20000))
    x = np.clip(x, -448, 448).astype(np.float32)
    mid = (o8.e4m3_values()[1:] + o8.e4m3_values()[:-1]) / 2      # ties
    x = np.concatenate([x, mid, -mid, [0.0, -0.0, 448.0, 2.0 ** -10, 2.0 ** -11]]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(o8.e4m3_encode(x), want)


@pytest.mark.parametrize("a,k", [(448.0, 0), (450.0, 1), (447.0, 0), (224.0, -1), (225.0, 0), (1.0, -8), (1.75, -8),
                                 (1.7578125, -7), (0.0, -100), (2.0 ** -120, -100), (448.0 * 2.0 ** -100, -100),
                                 (450.0 * 2.0 ** -100, -99), (3e38, 120)])
def test_scales_at_their_borders(a, k):
    x = np.zeros((16, 64))
    x[3, 5] = -a
    assert o8.block_scale(x) == 2.0 ** k


def test_block_error_is_half_a_step():
    x = np.random.default_rng(2).standard_normal((16, 128))
    code, s = o8.encode_block(x)
    y = o8.e4m3_decode(code) * s
    assert (np.abs(y - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * s)).all()
    x[2, 2] = np.inf
    code, s = o8.encode_block(x)
    assert np.isnan(s) and not code.any()


def test_layouts_are_permutations():
    code = np.arange(16 * 64).reshape(16, 64)
    for place in (o8.place_k, o8.place_v):
        got = place((code % 251).astype(np.uint8))
        assert sorted(got.tolist()) == sorted((code % 251).reshape(-1).tolist())
    k = o8.place_k((code // 64).astype(np.uint8))      # slots: 8 rows of 16 bytes, then the next 16 dims
    assert k[:128].reshape(8, 16).tolist() == [[t] * 16 for t in range(8)] and k[512] == 8
    v = o8.place_v((code // 64).astype(np.uint8))
    assert v[:16].tolist() == list(range(16))


def test_attend_is_causal_softmax():
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn((n, h, 64), generator=g, dtype=torch.float64) for n, h in ((3, 4), (21, 2), (21, 2)))
    mask = torch.arange(21)[None] <= torch.arange(18, 21)[:, None]
    want = torch.nn.functional.scaled_dot_product_attention(
        q.transpose(0, 1), k.transpose(0, 1).repeat_interleave(2, 0), v.transpose(0, 1).repeat_interleave(2, 0),
        attn_mask=mask)
    np.testing.assert_allclose(o8.attend(q.numpy(), k.numpy(), v.numpy()), want.transpose(0, 1).numpy(), rtol=1e-12, atol=1e-12)
