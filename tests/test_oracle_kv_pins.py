"""The oracle of the key/value cache against closed forms and brute force."""
import numpy as np
import pytest

from oracle import kv_cache as kv


def test_rotation_keeps_lengths_and_differences():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 1, 32))
    freq = 10000.0 ** (-np.arange(16) / 16)
    for neighbours in (False, True):
        turn = lambda x, p: kv.norm_rope(x, [p], freq, neighbours=neighbours, hadamard=True)  # noqa: E731
        assert np.isclose((turn(q, 7) ** 2).sum(), (q ** 2).sum())
        assert np.isclose((turn(q, 17) * turn(k, 12)).sum(), (turn(q, 105) * turn(k, 100)).sum())
    one = kv.norm_rope(np.eye(4)[None, :1], [np.pi / 2], [1.0, 0.0])
    assert np.allclose(one, [[[0, 0, 1, 0]]])
    assert np.allclose((kv.norm_rope(rng.standard_normal((3, 2, 64)), None, None, eps=0.0) ** 2).mean(-1), 1)


def test_bf16_below():
    for v, want in ((1.0, 1.0), (1.001, 1.0), (-1.001, -1.0078125), (0.0, 0.0), (-0.0, 0.0), (2.0 ** -133, 2.0 ** -133),
                    (-(2.0 ** -140), -(2.0 ** -133)), (2.0 ** -140, 0.0), (300.0, 300.0), (301.0, 300.0)):
        assert kv.bf16_below(v) == want and not np.signbit(kv.bf16_below(v)) == (want >= 0)


@pytest.mark.parametrize("seed", range(4))
def test_quantiser_covers_the_range_with_half_a_step(seed):
    x = np.random.default_rng(seed).standard_normal((50, 128)).astype(np.float32).astype(np.float64) * 10.0 ** seed
    codes, scale, off = kv.quantize(x)
    back = scale * codes + off
    assert (np.abs(back - x) <= scale * 0.5001).all() and codes.max() == 15
    assert (codes.min(-1) == 0).all() and (off <= x.min(-1, keepdims=True)).all()
    assert (scale <= (x.max(-1, keepdims=True) - off) / 15 * (1 + 2.0 ** -7)).all()
    grid = np.arange(16.0)
    codes, scale, off = kv.quantize(grid)
    assert (codes == grid).all() and scale == 1 and off == 0
    codes, scale, off = kv.quantize(np.array([3.0, 3.0]))
    assert (codes == 0).all() and scale == 0 and off == 3
    assert np.isnan(kv.quantize(np.array([1.0, np.inf]))[1]).all()


def test_pages_hold_what_was_written():
    rng = np.random.default_rng(1)
    c = kv.Cache(5, 2, 64, 32, [[3, 0], [4, -1]], [50, 20])
    want = {}
    for b, n in enumerate((50, 20)):
        for h in range(2):
            for slot in range(n):
                for second in (0, 1):
                    want[b, h, slot, second] = c.write(b, h, slot, second, rng.standard_normal(64))
    for (b, h, slot, second), v in want.items():
        codes, s, o = c.raw(b, h, slot, second)
        assert np.abs(s * codes + o - v).max() <= 1e-6 * np.abs(v).max()
    assert not c.pages[1].any() and not c.pages[2].any()
    assert c.place(1, 40) is None and c.place(0, 33) == (0, 0, 1)
    # token 17 of a page, its value codes: one group of 16 (64 + 8) bytes on, behind the keys' codes and parameters
    assert (c.pages[3, 1, 16 * 72 + 16 * 36 + 32:16 * 72 + 16 * 36 + 64] == c._at(0, 1, 17, 1)[0]).all()


def test_attention_is_a_mean_of_values():
    rng = np.random.default_rng(2)
    c = kv.Cache(2, 1, 64, 16, [[0, 1]], [20])
    for slot in range(20):
        c.write(0, 0, slot, 0, np.full(64, 0.5))
        c.write(0, 0, slot, 1, rng.standard_normal(64))
    r = kv.attention(c, 0, 0, rng.standard_normal((3, 2, 64)), 0.3)
    v = c.exact(0, 0, 20, 1)[0]
    for i in range(3):
        assert np.allclose(r["out"][i], v[:18 + i].mean(0)) and np.allclose(r["p"][i].sum(-1), 1)
        assert (r["p"][i, :, 18 + i:] == 0).all()
    assert np.isneginf(kv.attention(c, 0, 0, np.zeros((22, 1, 64)), 1.0)["lse"][:2]).all()


def test_eviction_by_hand():
    assert kv.evict(np.array([1, 5, 2, 9, 0, 3.]), np.arange(6), 6, 3, 1).tolist() == [3, 1, 5]
    assert kv.evict(np.array([1, 1, 1, 1.]), np.arange(4), 4, 2, 0).tolist() == [0, 1]
    assert kv.evict(np.array([1, np.nan, 1, 1.]), np.arange(4), 4, 3, 0).tolist() == [0, 3, 2]
    assert kv.evict(np.zeros(3), np.arange(3), 3, 5, 0).tolist() == [0, 1, 2]
