"""The ways that attention over a caller's pages distributes its work, at head_dim 128: each is reached, and right (needs a B200)."""
import numpy as np
import pytest

from tests import cache_helpers as H
from tests.test_gpu_cache import _attention_case, _lengths

pytestmark = pytest.mark.gpu

# sequences, k, mask blocks, longest, window, sinks; how the call goes over bf16 pages and over 4-bit ones, as 148 SMs have it
CASES = [
    (6, 8, True, 4000, 0, 0, "planned", "planned"),              # few ragged sequences: key ranges are cut
    (6, 8, True, 4000, 2500, 70, "planned", "planned"),          # ... within a window of most of it
    (30, 8, True, 900, 0, 0, "direct", "planned"),               # one to two tiles per SM: one stream per CTA; over codes planned
    (30, 8, True, 900, 300, 5, "direct", "planned"),
    (40, 8, True, 2700, 0, 0, "planned", "planned"),             # nearly as many units as SMs: two items per SM
    (60, 8, True, 2700, 0, 0, "planned", "planned"),             # units enough: pairs of tiles, not cut
    (60, 8, True, 2700, 2500, 1, "planned", "planned"),
    (2, 300, False, 2600, 0, 0, "planned", "planned"),           # two sequences' causal rows
    (1, 16, True, 3500, 0, 0, "direct", "direct")]               # one sequence: cut evenly


@pytest.mark.parametrize("kv4", [True, False])
@pytest.mark.parametrize("Hq,Hkv", [(12, 2), (8, 2)])
@pytest.mark.parametrize("n_seqs,k,blocks,longest,window,sinks,bf16_goes,codes_go", CASES)
def test_ways_to_distribute_work_of_wide_heads(kv4, Hq, Hkv, n_seqs, k, blocks, longest, window, sinks, bf16_goes, codes_go):
    t = H.lib_context(128, Hq, Hkv, n_seqs * k * (k + 1 if blocks else 1))
    rng = np.random.default_rng(n_seqs + k)
    ns = _lengths(rng, n_seqs, longest) if n_seqs > 2 else [longest] + [longest // 3] * (n_seqs - 1)

    def outside_the_pool(table, c):
        table[n_seqs // 2 if n_seqs > 2 else 0, [0, 7, 13]] = [-1, len(c.pools[0]), 2 ** 31 - 1]
        table[0, 0] = -3 if n_seqs % 4 else table[0, 0]
    _attention_case(t, kv4, 128, Hq, Hkv, k, blocks, ns, window, sinks, 81 + n_seqs, fused=n_seqs % 4 == 2, spoil=outside_the_pool)
    # (a plan notes its tiles; -1 says that every CTA worked out its own item)
    assert ("direct" if t.attention_route()[2] < 0 else "planned") == (codes_go if kv4 else bf16_goes)
    t.close()
