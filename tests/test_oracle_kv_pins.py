"""The oracle of heads, cache and attention, held to values worked out by hand."""
import numpy as np
import pytest

from oracle import kv

ONE, TWO, HALF, MINUS = 0x3F80, 0x4000, 0x3F00, 0xBF80


def patterns(x):
    return kv.round_bf16(np.asarray(x, dtype=np.float64))


def test_rounding_to_bf16_is_to_nearest_even():
    assert list(patterns([1.0, 1.00390625, 1.01171875, -2.0, 0.0])) == [0x3F80, 0x3F80, 0x3F82, 0xC000, 0]
    assert kv.round_bf16(np.nan) == 0x7FC0 and kv.round_bf16(np.inf) == 0x7F80


def test_norm_of_a_head():
    x = np.tile(np.array([3, 4], dtype=np.float64), 8).reshape(1, 1, 16)                 # mean square 12.5
    y = kv.turn(patterns(x), rmsnorm=True, eps=0.0)
    np.testing.assert_allclose(y, x / np.sqrt(12.5), rtol=1e-15)
    y = kv.turn(patterns(x), rmsnorm=True, gain=np.full(16, TWO, dtype=np.uint16), eps=12.5)
    np.testing.assert_allclose(y, 2 * x / 5, rtol=1e-15)


@pytest.mark.parametrize("interleaved", (False, True))
def test_rotation_by_a_quarter_turn(interleaved):
    x = np.arange(1, 33, dtype=np.float64).reshape(1, 1, 32)
    y = kv.turn(patterns(x), positions=[2], inv_freq=np.full(8, np.pi / 4), rotary_dim=16, interleaved=interleaved)[0, 0]
    l, r = (np.arange(0, 16, 2), np.arange(1, 16, 2)) if interleaved else (np.arange(8), np.arange(8, 16))
    np.testing.assert_allclose(y[l], -x[0, 0, r], atol=1e-5)                              # (pi / 4 is a 32-bit number)
    np.testing.assert_allclose(y[r], x[0, 0, l], atol=1e-5)
    assert np.array_equal(y[16:], x[0, 0, 16:])


def codebook():
    return patterns(np.arange(-8, 8) / 8.0 + 1 / 16)                                      # -15/16, -13/16, ... 15/16: boundaries at k / 8


def test_a_value_on_a_boundary_goes_to_the_lower_centroid():
    assert np.array_equal(kv.boundaries(codebook()), np.arange(-7, 8) / 8.0)
    x = np.zeros(64)
    x[:5] = [2.0, 0.25, 0.26, -1.75, -2.0]                                                # scale 2: 1, 0.125, 0.13, -0.875, -1
    idx, scale = kv.quantize(patterns(x), codebook())
    assert scale.tolist() == [TWO]
    assert idx[:6].tolist() == [15, 8, 9, 0, 0, 7]                                        # (0 is a boundary too)
    v = kv.values(idx, scale, codebook())
    assert v[:5].tolist() == [2 * 15 / 16, 2 * 1 / 16, 2 * 3 / 16, -2 * 15 / 16, -2 * 15 / 16]


def test_blocks_of_zeros_and_of_infinities():
    idx, scale = kv.quantize(np.zeros(128, dtype=np.uint16), codebook())
    assert not scale.any() and (idx == 7).all()
    x = np.zeros(64, dtype=np.uint16)
    x[3], x[7] = 0xFF80, 0x7FC1
    assert kv.quantize(x, codebook())[1].tolist() == [0x7FC1]


@pytest.mark.parametrize("D", (64, 128, 256))
def test_pages_use_every_byte_once(D):
    pages = kv.Pages(2, 32, 3, D)
    count = np.zeros((pages.bytes.size, 2), dtype=int)
    for page in range(2):
        for token in range(32):
            ka, ks, va, vs, sa = pages.places(page, token)
            for a, s in ((ka, ks), (va, vs)):
                np.add.at(count, (a, np.broadcast_to(s // 4, a.shape)), 1)
            for h in range(2):
                np.add.at(count, (sa + h, np.zeros_like(sa)), 1)
                np.add.at(count, (sa + h, np.ones_like(sa)), 1)
    assert (count == 1).all()


def test_pages_give_back_what_was_written():
    g = np.random.default_rng(1)
    books = np.stack([codebook(), patterns(np.sort(g.uniform(-1, 1, 16)))])
    pages = kv.Pages(3, 32, 2, 128, fill=g.integers(0, 256, 3 * 2 * 2 * 17 * 128))
    rows = {}
    for page, token in ((1, 5), (1, 6), (2, 31), (1, 21), (0, 0)):
        k, v = patterns(g.standard_normal((2, 128))), patterns(g.standard_normal((2, 128)))
        pages.write(page, token, k, v, books)
        rows[page, token] = k, v
    for (page, token), (k, v) in rows.items():
        got = pages.read(page, token, books)
        for x, y, b in ((k, got[0], books[0]), (v, got[1], books[1])):
            assert np.array_equal(kv.values(*kv.quantize(x, b), b), y)
    # a byte of the documented layout by hand: token 5 of page 1, head 1, element 70 of K (even: low nibble) and 84 of V (84 % 32 >= 16: high)
    tile = ((1 * 2 + 1) * 2 + 0) * 17 * 128
    k, v = rows[1, 5]
    assert pages.bytes[tile + ((70 // 16 % 4) * 16 + 5) * 16 + 8 + 6 // 2] & 15 == kv.quantize(k, books[0])[0][1, 70]
    assert pages.bytes[tile + 8 * 128 + (1 * 16 + 84 % 16) * 16 + 2 * 4 + 1] >> 4 == kv.quantize(v, books[1])[0][1, 84]


def test_attention_of_two_tokens():
    k = np.zeros((2, 1, 64))
    k[0, 0, 0], k[1, 0, 0] = 1.0, 2.0
    v = np.stack([np.full((1, 64), 1.0), np.full((1, 64), 5.0)])
    q = np.zeros((2, 2, 64), dtype=np.uint16)
    q[:, 0, 0] = ONE
    there = np.array([True, True])
    out, lse, spread, size = kv.attention(q, k, v, there, 2, np.log(3.0))
    np.testing.assert_allclose(out[0], 1.0)                                               # row 0 sees token 0 alone
    np.testing.assert_allclose(out[1, 0], (3 * 1 + 9 * 5) / 12)
    np.testing.assert_allclose(out[1, 1], 3.0)                                            # a query of zeros: the mean
    np.testing.assert_allclose(lse[1], [np.log(12.0), np.log(2.0)])
    np.testing.assert_allclose(size[1], [2 * np.log(3.0), 0])
    out, lse, _, _ = kv.attention(q, k, v, there, 2, np.log(3.0), causal=False)
    np.testing.assert_allclose(out[0, 0], 4.0)
    out, lse, _, _ = kv.attention(q, k, v, there, 2, np.log(3.0), window=1)
    np.testing.assert_allclose(out[1, 0], 5.0)
    out, lse, _, _ = kv.attention(q, k, v, np.array([False, True]), 2, 1.0)
    assert not out[0].any() and np.isneginf(lse[0]).all()
    out, lse, _, _ = kv.attention(q, k[:1], v[:1], there[:1], 1, 1.0)                     # two rows, one token: the first stands before it
    assert not out[0].any() and np.isneginf(lse[0]).all() and (out[1] == 1).all()


def test_positions_that_are_not_in_the_cache():
    assert kv.place([4, 7], 32, 8, 33) == (7, 1)
    assert kv.place([4, 7], 32, 7, 33) is None and kv.place([-1], 32, 7, 3) is None
    assert kv.place([4], 32, 8, 32) is None and kv.place([4], 32, 8, -1) is None
