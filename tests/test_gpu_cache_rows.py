"""Rows held in 4 bits where 32-bit arithmetic is at its limits, byte by byte against the plain statement in 64 bits (needs a B200)."""
import numpy as np
import pytest
import torch

from tests import cache_helpers as H

pytestmark = pytest.mark.gpu


def _groups_are_stored_as_stated(groups):
    """Stores groups [n, 32] (bf16 values, as float64) as rows of one head of 64 dimensions, K as they are and V reversed; the records' bytes are the statement's."""
    from paper_2511_08923_b200 import kv4_pages
    groups = np.asarray(groups, dtype=np.float64)
    assert np.array_equal(groups, H.bf16_round(groups))
    groups = np.concatenate([groups, groups[:len(groups) % 2]])
    x = groups.reshape(-1, 64)
    n_pages = (len(x) + 63) // 64
    x = np.concatenate([x, np.zeros((n_pages * 64 - len(x), 64))])
    t = H.lib_context(64, 1, 1, 0)
    pools = [kv4_pages(n_pages, 1, 64) for _ in range(2)]
    k, v = (torch.from_numpy(np.ascontiguousarray(r)[:, None]).to(torch.bfloat16).cuda() for r in (x, x[::-1]))
    t.kv4_store(k, v, torch.arange(len(x), dtype=torch.int32, device="cuda:0"), *pools)
    t.sync()
    for rows, pool in ((x, pools[0]), (x[::-1], pools[1])):
        want = H.records(rows.reshape(n_pages, 1, 64, 64))
        assert np.array_equal(pool.cpu().numpy(), want), np.argwhere(pool.cpu().numpy() != want)[:8]
    t.close()


def test_codes_at_the_top_of_the_range():
    """Groups from -2^126 to 2^126: an element's distance from the base exceeds the largest float.  All 128 bf16 numbers of the topmost binade, of either sign."""
    top = 2.0 ** 126
    binade = top / 2 * (1 + np.arange(128) / 128)
    values = np.concatenate([binade, -binade, binade / 2, [0.9 * top - 0.9 * top % 2.0 ** 118, 0.0]])
    values = np.concatenate([values, np.zeros(-len(values) % 30)]).reshape(-1, 30)
    ends = np.tile([[-top, top]], (len(values), 1))
    _groups_are_stored_as_stated(np.concatenate([ends, values], 1))
    _groups_are_stored_as_stated(np.concatenate([ends * [1, 0.5], np.clip(values, -top, top / 2)], 1))


@pytest.mark.parametrize("exponent", [-100, -98, -60, 0, 50, 90, 105])
@pytest.mark.parametrize("mantissa", [1.0, 1.5])
def test_codes_of_elements_next_to_the_border_between_two(exponent, mantissa):
    """Where an element is far smaller than its group's scale, its distance from the base does not fit 32 bits; a border lies at 0 for these groups, so that such
    an element's sign alone decides (0 itself is a tie)."""
    s = mantissa * 2.0 ** exponent
    groups = []
    for r in range(16, 31):                                      # base -(r + 1/2) s: the border between r and r + 1 is at 0
        lo = -(r - 15.5) * s
        g = np.linspace(lo, lo + 15 * s, 32)
        g = H.bf16_round(g)
        for tiny in ([2.0 ** -25, 2.0 ** -30 * (1 + 2.0 ** -7), 2.0 ** -33], [2.0 ** -17, 2.0 ** -18 * (1 + 2.0 ** -7), 2.0 ** -18], [2.0 ** -19, 2.0 ** -19 * (1 + 2.0 ** -7), 2.0 ** -20],
                     [2.0 ** -20 * (1 + 2.0 ** -7), 2.0 ** -21, 2.0 ** -22]):
            tiny = np.array(tiny) * 2.0 ** exponent
            g[3:10] = np.concatenate([tiny, -tiny, [0.0]])
            groups.append(g.copy())
            c, scale, base = H.quantise(g)
            assert scale == s and base == -(r + 0.5) * s and len(set(c[3:9].tolist())) == 2
    _groups_are_stored_as_stated(groups)


def test_codes_of_very_small_groups():
    """Scales and spreads on both sides of 1e-30, below which quotients are divisions; numbers of few bits among them, so that ties are."""
    rng = np.random.default_rng(3)
    groups = []
    for exponent in range(-112, -90):
        x = rng.standard_normal((12, 32))
        x[6:] = np.rint(x[6:] * 8) / 4
        x[np.abs(x) < 2.0 ** -12] = 0                            # (normal numbers, for the plain statement)
        groups.append(H.bf16_round(x * 2.0 ** exponent))
    groups = np.concatenate(groups)
    s = H.quantise(groups)[1]
    assert s.min() < 2.0 ** -110 and (s > 1.2e-30).any() and (s > 1e-32).any()
    _groups_are_stored_as_stated(groups)
