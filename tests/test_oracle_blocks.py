"""Pins of the decoder block's oracle: finite differences, closed forms, published vectors of the generator."""
import numpy as np
import pytest

from oracle import block_oracle as blk


@pytest.mark.parametrize("cap,bias,causal,prefix", [(0.0, False, False, None), (0.0, True, True, None), (3.0, False, True, [2, 0]), (2.0, True, False, None)])
def test_attention_gradient_is_that_of_differences(cap, bias, causal, prefix):
    rng = np.random.default_rng(1)
    M, heads, kv, dim, begin = 9, 4, 2, 3, [1, 6, 8]
    x, dy = rng.normal(size=(M, (heads + 2 * kv) * dim)), rng.normal(size=(M, heads * dim))
    slopes = rng.normal(size=heads) if bias else None
    see = blk.visible(M, begin, causal, prefix)
    f = lambda t: (blk.attention(t, heads, kv, dim, see, None, cap, slopes)[0] * dy).sum()  # noqa: E731
    dx = blk.attention(x, heads, kv, dim, see, None, cap, slopes, dy)[2]
    num = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        for sign in (1, -1):
            t = x.copy()
            t[i] += sign * 1e-5
            num[i] += sign * f(t) / 2e-5
    assert np.abs(num - dx).max() < 1e-7 * max(1, np.abs(dx).max())
    assert not dx[0].any() and not dx[8].any()                           # rows of no sequence


def test_attention_of_equal_keys_is_the_mean_and_masks_do_what_they_say():
    M, dim = 7, 2
    x = np.zeros((M, 3 * dim))
    x[:, 2 * dim:] = np.arange(M)[:, None]
    see = blk.visible(M, [0, 4, 4, 6], True, [2, 5, 0])
    y = blk.attention(x, 1, 1, dim, see)[0][:, 0]
    assert y.tolist() == [0.5, 0.5, 1.0, 1.5, 4.0, 4.5, 0.0]


def test_rotary_keeps_lengths_and_relative_angles_and_goes_back():
    rng = np.random.default_rng(2)
    M, dim = 5, 8
    x = rng.normal(size=(M, 3 * dim))
    for adjacent in (False, True):
        for own in (False, True):
            pos = np.stack([np.arange(M) + 3, np.arange(M)[::-1]])
            y, _ = blk.rotary(x, 1, 1, dim, (2, 1), pos, 100.0, adjacent, own)
            assert np.allclose((y ** 2).sum(1), (x ** 2).sum(1))
            assert np.array_equal(y[:, 2 * dim:], x[:, 2 * dim:])
            b, _ = blk.rotary(y, 1, 1, dim, (2, 1), pos, 100.0, adjacent, own, back=True)
            assert np.allclose(b, x)
    # a score depends on the difference of the positions only
    one = lambda t: blk.rotary(np.tile(x[:1], (M, 1)), 1, 1, dim, (4,), [np.arange(M) + t], 100.0)[0]  # noqa: E731
    a, b = one(0), one(1000)
    assert np.allclose(a[:, :dim] @ a[:, dim:2 * dim].T, b[:, :dim] @ b[:, dim:2 * dim].T)


@pytest.mark.parametrize("kind", [1, 2, 3])
def test_gated_gradient_is_that_of_differences(kind):
    rng = np.random.default_rng(3)
    x, W, b, dy = rng.normal(size=(4, 3)), rng.normal(size=(3, 10)), rng.normal(size=10), rng.normal(size=(4, 5))
    r = blk.gated(x, W, b, kind, dy, 0.0)
    for name, v in (("dx", x), ("dW", W), ("db", b)):
        num = np.zeros_like(v)
        for i in np.ndindex(*v.shape):
            keep = v[i]
            for sign in (1, -1):
                v[i] = keep + sign * 1e-6
                num[i] += sign * (blk.gated(x, W, b, kind, dy, 0.0)["y"][0] * dy).sum() / 2e-6
            v[i] = keep
        assert np.abs(num - r[name][0]).max() < 1e-6


def test_generator_gives_the_published_words():
    """Known answers of Philox4x32-10 (the generator's authors' test vectors)."""
    f = 0xFFFFFFFF
    assert blk.philox((0, 0, 0, 0), (0, 0)) == (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)
    assert blk.philox((f, f, f, f), (f, f)) == (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)
    assert blk.philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)
    k = blk.kept(0, 40000, 0.3, 12345678901234567890, 7, 2)
    assert abs(k.mean() - 0.7) < 4 * np.sqrt(0.3 * 0.7 / 40000)
