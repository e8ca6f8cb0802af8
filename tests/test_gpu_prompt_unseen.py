"""Keys and values that a query does not see have no effect on it, not on a bit: queries of the same wave before a changed key, in later tiles, and with the keys
in parts."""
import numpy as np
import pytest

from launch_rules import prompt_cut
from prompt_cases import PromptCase

pytestmark = pytest.mark.gpu


def _changed(c, row, factor):
    """The result with one key and value changed, as the device holds them."""
    k, v = c.k[row].copy(), c.v[row].copy()
    c.k[row], c.v[row] = np.float32(factor) * k, np.float32(-factor) * v
    got = c.run()
    c.k[row], c.v[row] = k, v
    return got


@pytest.mark.parametrize("dtype,H,H_kv,d_k", [("bf16", 4, 2, 64), ("bf16", 2, 2, 128), ("bf16", 1024, 8, 64), ("bf16", 2, 2, 192), ("f32", 2, 2, 64), ("f32", 2, 1, 128),
                                              ("f32", 2, 2, 32), ("f32", 1, 1, 256)])
def test_queries_before_a_changed_key(dtype, H, H_kv, d_k):
    """A key that scores far above the others moves the reference of the queries that see it, and of no other."""
    n = 230
    c = PromptCase([n], [n], H, H_kv, d_k, dtype, seed=d_k + H)
    clean = c.run()
    for row in (33, 66, 100, 110, 127, 150, 200, 229):
        for factor in (8.0, 64.0, np.inf, np.nan):
            got = _changed(c, row, factor)
            assert np.array_equal(got[:row], clean[:row]), (row, factor)
            assert factor > 8 or not np.array_equal(got[row:], clean[row:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,d_k", [(2, 64), (1, 128)])
def test_queries_before_a_changed_key_with_keys_in_parts(dtype, H, d_k):
    n_q, n_k = 20, 3000
    assert prompt_cut(dtype, 1, n_q, n_k, H, H, d_k)[1] > 1
    c = PromptCase([n_q], [n_k], H, H, d_k, dtype, seed=2)
    clean = c.run()
    for i in (1, 7, 16, 19):                                     # the first query that sees the key
        for factor in (16.0, np.inf, np.nan):
            got = _changed(c, n_k - n_q + i, factor)
            assert np.array_equal(got[:i], clean[:i]), (i, factor)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_finite_with_keys_in_parts(dtype):
    """NaN and infinities in keys and values that some queries see, and that none does, in several parts of the keys."""
    n_q, n_k, H, d_k = 20, 3000, 2, 64
    c = PromptCase([n_q], [n_k], H, H, d_k, dtype, seed=6, tail=70)
    clean = c.run()[:n_q]
    c.k[n_k:], c.v[n_k:] = np.nan, np.inf                        # (rows of no sequence)
    assert np.array_equal(c.run()[:n_q], clean)
    c.v[n_k - 5, 3::7] = np.nan                                  # values that the last five queries see
    c.v[n_k - 2, 4::7] = np.inf
    got, cols = c.run()[:n_q], np.arange(H * d_k)
    assert np.array_equal(got[:15], clean[:15])
    odd = np.zeros((n_q, H * d_k), dtype=bool)
    odd[15:, 3::7] = True
    odd[18:, 4::7] = True
    assert not np.isfinite(got[odd]).any() and np.isfinite(got[~odd]).all()
    rest = np.delete(cols, np.r_[3:H * d_k:7, 4:H * d_k:7])
    e = PromptCase([n_q], [n_k], H, H, d_k, dtype, seed=6, tail=70)
    want, bound = e.expected(0)
    assert (np.abs(got - want) <= bound)[:, rest].all()          # (in the other columns all is finite)
    for row in (0, 700, 2000, n_k - n_q):                        # a key that every query sees, in the first, a middle and the last part
        d = PromptCase([n_q], [n_k], H, H, d_k, dtype, seed=6, tail=70)
        d.k[row, :d_k] = np.nan
        got = d.run()[:n_q]
        assert np.isnan(got[:, :d_k]).all() and (np.abs(got - want) <= bound)[:, d_k:].all(), row
        d = PromptCase([n_q], [n_k], H, H, d_k, dtype, seed=6, tail=70)
        d.v[row, d_k + 1] = -np.inf
        got = d.run()[:n_q]
        assert not np.isfinite(got[:, d_k + 1]).any() and np.delete(np.abs(got - want) <= bound, d_k + 1, 1).all(), row
