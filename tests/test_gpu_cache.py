"""Operators over a paged cache that the caller keeps, against plain statements in 64 bits (needs a B200)."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests import cache_helpers as H

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda:0")


# ---- page map ---------------------------------------------------------------
def _map_case(t, n, m, held, free, begin, table, max_rows, in_place=False):
    want = H.page_map(n, m, held, free, begin, table, max_rows)
    d = dict(n=_i32(n), m=_i32(m), held=_i32(held), free=_i32(free), table=_i32(table))
    held_out = d["held"] if in_place else torch.full_like(d["held"], -7)
    starts, slots = torch.full((len(n) + 1,), -7, dtype=torch.int32, device="cuda:0"), torch.full((max_rows + 5,), -7, dtype=torch.int32, device="cuda:0")
    counts = torch.full((3,), begin, dtype=torch.int32, device="cuda:0")
    out_counts = counts if in_place else torch.full((3,), -7, dtype=torch.int32, device="cuda:0")
    t.page_map(d["n"], d["m"], d["held"], d["free"], d["table"], held_out, starts, slots[:max_rows], out_counts, free_begin=counts[:1] if begin or in_place else None)
    t.sync()
    for what, got, ref in zip(("table", "held", "starts", "slots", "counts"), (d["table"], held_out, starts, slots[:max_rows], out_counts), want):
        assert np.array_equal(got.cpu().numpy(), ref), what
    assert (slots[max_rows:] == -7).all()
    return want


def _table(rng, held, width, n_pages):
    table = np.full((len(held), width), -1, dtype=np.int32)
    pages = rng.permutation(n_pages)
    at = 0
    for i, h in enumerate(held):
        h = min(h, width)
        table[i, :h] = pages[at:at + h]
        at += h
    return table, pages[at:].astype(np.int32)


@pytest.mark.parametrize("impl", [0, 1])
@pytest.mark.parametrize("n_seqs,n_hi,m_hi", [(1, 0, 1), (1, 63, 1), (1, 64, 64), (5, 200, 16), (33, 300, 0), (513, 100, 9), (700, 5000, 150), (4096, 70, 3)])
def test_page_map_against_a_plain_one(impl, n_seqs, n_hi, m_hi):
    t = H.lib_context(64, 4, 2, 0, impl=impl)
    rng = np.random.default_rng(n_seqs + n_hi)
    n = rng.integers(0, n_hi + 1, n_seqs)
    n[rng.random(n_seqs) < 0.2] = -1 - int(rng.integers(0, 9))
    m = rng.integers(-2, m_hi + 1, n_seqs)
    held = np.where(n < 0, rng.integers(0, 3, n_seqs), (np.maximum(n, 0) + 63) // 64 + (rng.random(n_seqs) < 0.3)).astype(np.int64)
    width = int(max(held.max(), (n_hi + max(m_hi, 0) + 63) // 64, 1))
    table, free = _table(rng, held, width, int(held.sum()) + n_seqs * 4 + 40)
    total = int(np.where(n >= 0, np.maximum(m, 0), 0).sum())
    for begin, max_rows, in_place in ((0, total + 3, False), (2, total, True), (0, max(total - 5, 0), False), (max(len(free) - 3, 0), total + 2100, True)):
        _map_case(t, n, m, held.copy(), free, begin, table.copy(), max_rows, in_place)
    t.close()


def test_page_map_when_the_table_or_the_list_ends():
    t = H.lib_context(64, 4, 2, 0)
    rng = np.random.default_rng(5)
    n, m, held = np.array([100, 500, 0, 128]), np.array([200, 10, 1, 0]), np.array([2, 4, 0, 2])
    table, free = _table(rng, held, 4, 20)                       # sequence 1 is longer than the table, sequence 0 outgrows it
    _map_case(t, n, m, held, free, 0, table, 260)
    _map_case(t, n, m, held, free[:1], 0, table, 260)            # one page for three
    _map_case(t, n, m, held, free[:0], 0, table, 260)
    _map_case(t, np.array([100, -1, 70, -9]), np.array([60, 5, 200, 5]), np.array([-3, -4, 9, 9]), free, 0, table, 260, True)       # counts of held pages that make no sense
    _map_case(t, np.array([2 ** 31 - 1]), np.array([300]), np.array([4]), free, 0, table[:1], 70)          # positions beyond 32 bits
    t.close()


def test_page_map_saturates():
    """Rows beyond 2^31 - 1 in all: the counters stop there; the slots that were asked for are right."""
    t = H.lib_context(64, 4, 2, 0)
    big = 2 ** 31 - 1
    n, m, held, table, free = _i32([0, 3, 5]), _i32([1, big, big]), _i32([0, 0, 0]), _i32(np.full((3, 2), -1)), _i32(np.arange(9))
    starts, slots, counts = _i32([0] * 4), _i32([0] * 200), _i32([0] * 3)
    t.page_map(n, m, held, free, table, held, starts, slots, counts)
    t.sync()
    assert starts.tolist() == [0, 1, big, big] and counts.tolist() == [5, big - 126, big] and held.tolist() == [1, 2, 2]
    assert table.tolist() == [[0, -1], [1, 2], [3, 4]]
    assert slots.tolist() == [0] + [64 + p if p < 64 else 64 + p for p in range(3, 128)] + [-1] * 74
    t.close()


# ---- rows in 4 bits ---------------------------------------------------------
def _rows(rng, rows, heads, hd):
    x = rng.standard_normal((rows, heads, hd)) * np.exp(rng.standard_normal((rows, heads, 1)) * 2)
    x = H.bf16_round(x + rng.standard_normal((rows, heads, 1)) * (rng.random((rows, 1, 1)) < 0.3) * 30)
    if rows > 3:
        x[1] = 0.75                                              # constant groups: scale 0, held exactly
        x[2, :, 32:64] = 0.0
        x[3, 0, :4] = [np.nan, np.inf, -np.inf, 3e38]
    return x


@pytest.mark.parametrize("hd,heads", [(64, 2), (128, 8), (128, 1), (64, 5)])
@pytest.mark.parametrize("rows,strided", [(1, False), (7, True), (130, False), (333, True)])
def test_store_and_load_rows_in_4_bits(hd, heads, rows, strided):
    from paper_2511_08923_b200 import kv4_page_bytes, kv4_pages
    t = H.lib_context(hd, heads, heads, 0)
    rng = np.random.default_rng(rows * hd + heads)
    n_pages = (rows + 63) // 64 + 2
    slots = rng.permutation(n_pages * 64)[:rows]
    skip = rng.random(rows) < 0.1
    slots[skip] = rng.choice([-1, -64, n_pages * 64, 2 ** 31 - 1], int(skip.sum()))
    k, v = _rows(rng, rows, heads, hd), _rows(rng, rows, heads, hd)
    both = torch.from_numpy(np.concatenate([k, v], 1)).to(torch.bfloat16).cuda()
    dk, dv = both[:, :heads], both[:, heads:]
    if not strided:
        dk, dv = dk.contiguous(), dv.contiguous()
    pools = [kv4_pages(n_pages, heads, hd) for _ in range(2)]
    for p in pools:
        p.fill_(0xA5)
    t.kv4_store(dk, dv, _i32(slots), *pools)
    back = torch.full((rows, 2 * heads + 1, hd), 7.0, dtype=torch.bfloat16, device="cuda:0")
    bk, bv = (back[:, :heads], back[:, heads:2 * heads])
    t.kv4_load(*pools, _i32(slots), bk, bv)
    t.sync()
    n_codes = 64 * hd // 2
    for x, pool, got in ((k, pools[0], bk), (v, pools[1], bv)):
        want = np.full((n_pages, heads, kv4_page_bytes(hd)), 0xA5, dtype=np.uint8)
        for r in np.nonzero(~skip)[0]:                           # a page holding this row alone, and its bytes
            page, place = divmod(int(slots[r]), 64)
            one = np.zeros((heads, 64, hd)); one[:, place] = x[r]
            rec = H.records(one)
            for group in range(hd // 32):
                at = (group * 64 + place) * 16
                want[page, :, at:at + 16] = rec[:, at:at + 16]
            at = n_codes + place * hd // 8
            want[page, :, at:at + hd // 8] = rec[:, at:at + hd // 8]
        assert np.array_equal(pool.cpu().numpy(), want)
        ref = np.where(skip[:, None, None], 7.0, H.values(*H.quantise(x)))
        assert np.array_equal(got.double().cpu().numpy(), ref)
        # half a step of the scale, a step at the ends for the scale's and the base's rounding, and the value's own rounding
        fine = np.isfinite(x) & (np.abs(x) < 1e30) & ~skip[:, None, None]
        s = np.repeat(H.quantise(x)[1], 32, -1)
        assert (np.abs(got.double().cpu().numpy() - np.where(fine, x, 0)) <= 1.0 * s + 2.0 ** -8 * np.abs(x))[fine].all()
    assert (back[:, 2 * heads] == 7.0).all()
    t.close()


# ---- attention --------------------------------------------------------------
def _attention_case(t, kv4, hd, Hq, Hkv, k, blocks, ns, window, sinks, seed, fused=False, spoil=None):
    B, T = len(ns), k * (k + 1) if blocks else k
    c = H.Cache(seed, kv4, hd, Hkv, k, ns)
    rng = np.random.default_rng(seed + 1)
    q = H.bf16_round(rng.standard_normal((B * T, Hq, hd)))
    kl, vl = (H.bf16_round(rng.standard_normal((B * k * k, Hkv, hd))) for _ in range(2)) if blocks else (None, None)
    table = c.table.copy()
    if spoil is not None:
        spoil(table, c)

    def dev(x):
        if x is None:
            return None
        d = torch.from_numpy(x).to(torch.bfloat16).cuda()
        if not fused:
            return d
        wide = torch.full((d.shape[0], d.shape[1] + 3, hd), float("nan"), dtype=torch.bfloat16, device="cuda:0")
        wide[:, 1:1 + d.shape[1]] = d
        return wide[:, 1:1 + d.shape[1]]
    dq, dkl, dvl = dev(q), dev(kl), dev(vl)
    if blocks:
        for i, n in enumerate(ns):
            if n < 0:                                            # nobody's local rows
                dkl[i * k * k:(i + 1) * k * k] = float("nan"); dvl[i * k * k:(i + 1) * k * k] = float("nan")
    out = torch.full((B * T + 1, Hq * hd), 5.0, dtype=torch.bfloat16, device="cuda:0")
    call = t.attention_kv4 if kv4 else t.attention_window
    call(dq, c.pools[0], c.pools[1], _i32(table), _i32(ns), dkl, dvl, out[:B * T], B, k, window=window, sinks=sinks)
    t.sync()
    got = out.double().cpu().numpy()
    assert (got[B * T] == 5.0).all()
    n_pages = len(c.pools[0])
    for i, n in enumerate(ns):
        mine = got[i * T:(i + 1) * T].reshape(T, Hq, hd)
        if n < 0:
            assert (mine == 5.0).all()
            continue
        vis = H.visible(n, k, blocks, window, sinks, n + k)
        for p in range((n + k + 63) // 64):
            if not 0 <= table[i, p] < n_pages:
                vis[:, p * 64:(p + 1) * 64] = False
        local = [x[i * k * k:(i + 1) * k * k] for x in (kl, vl)] if blocks else [None, None]
        ref, spread = H.attention(q[i * T:(i + 1) * T], c.K[i], c.V[i], vis, k, *local)
        assert np.isfinite(mine).all(), i
        worst = (np.abs(mine - ref) - H.tolerance(ref, spread)).max()
        assert worst <= 0, (i, n, worst, np.abs(mine - ref).max())
    return got


HEADS = [(64, 4, 2), (128, 8, 2), (128, 12, 2), (128, 4, 4), (128, 7, 1), (64, 20, 1)]
IMPLS = [1, 0]


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("kv4", [True, False])
@pytest.mark.parametrize("hd,Hq,Hkv", HEADS)
def test_single_tokens(impl, kv4, hd, Hq, Hkv):
    t = H.lib_context(hd, Hq, Hkv, 64, impl=impl)
    _attention_case(t, kv4, hd, Hq, Hkv, 1, False, [0, 1, 62, 63, 64, 65, 127, 200, 700], 0, 0, 11)
    _attention_case(t, kv4, hd, Hq, Hkv, 1, False, [0, 5, 63, 64, 130, 600, 999], 100, 4, 12, fused=True)
    _attention_case(t, kv4, hd, Hq, Hkv, 1, False, [300, 64], 1, 0, 13)                  # itself alone
    _attention_case(t, kv4, hd, Hq, Hkv, 1, False, [300, 700, 10], 64, 70, 14)           # sinks reach into the second page
    _attention_case(t, kv4, hd, Hq, Hkv, 1, False, [1500], 0, 0, 15)
    t.close()


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("kv4", [True, False])
@pytest.mark.parametrize("hd,Hq,Hkv", HEADS)
def test_steps(impl, kv4, hd, Hq, Hkv):
    t = H.lib_context(hd, Hq, Hkv, 300, impl=impl)
    _attention_case(t, kv4, hd, Hq, Hkv, 4, True, [0, 1, 63], 0, 0, 21)
    _attention_case(t, kv4, hd, Hq, Hkv, 4, True, [64, 65, 127], 30, 2, 22, fused=True)
    _attention_case(t, kv4, hd, Hq, Hkv, 2, True, [0, 400, 60], 50, 1, 23)
    _attention_case(t, kv4, hd, Hq, Hkv, 1, True, [0, 9, 333], 3, 0, 24)
    _attention_case(t, kv4, hd, Hq, Hkv, 5, True, [300, 3], 2, 0, 25)                    # a window shorter than the block
    _attention_case(t, kv4, hd, Hq, Hkv, 8, True, [500, 59], 130, 65, 26)
    t.close()


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("kv4", [True, False])
@pytest.mark.parametrize("n,window,sinks", [(1100, 0, 0), (1100, 300, 4), (2300, 640, 0)])
def test_steps_of_16(impl, kv4, n, window, sinks):
    t = H.lib_context(128, 8, 2, 272, impl=impl)
    _attention_case(t, kv4, 128, 8, 2, 16, True, [n], window, sinks, 27)
    t.close()


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("kv4", [True, False])
@pytest.mark.parametrize("hd,Hq,Hkv", [(64, 4, 2), (128, 12, 2)])
def test_causal_chunks(impl, kv4, hd, Hq, Hkv):
    t = H.lib_context(hd, Hq, Hkv, 400, impl=impl)
    _attention_case(t, kv4, hd, Hq, Hkv, 200, False, [0, 77], 0, 0, 31)
    _attention_case(t, kv4, hd, Hq, Hkv, 129, False, [250, 1], 70, 3, 32, fused=True)
    _attention_case(t, kv4, hd, Hq, Hkv, 3, False, [61, 0, 500], 0, 0, 33)
    t.close()


def _lengths(rng, n_seqs, longest):
    ns = [int(x) for x in rng.integers(0, 130, n_seqs)]
    ns[n_seqs // 2], ns[1] = longest, -1
    return ns


@pytest.mark.parametrize("kv4", [True, False])
@pytest.mark.parametrize("n_seqs,k,blocks,longest,window,sinks", [
    (40, 8, True, 900, 0, 0),             # more tiles than SMs, few pages: two CTAs per SM where pages are loaded whole
    (40, 8, True, 2700, 0, 0),            # ... many pages: planned
    (40, 8, True, 2700, 500, 70),         # ... within a window
    (60, 5, True, 3000, 0, 0),            # tiles of ragged lengths, cut key ranges
    (6, 16, True, 4000, 0, 0),
    (280, 5, True, 500, 100, 1),          # more units than are planned
    (300, 1, False, 700, 0, 0),
    (2, 70, False, 2600, 0, 0),           # two sequences' causal rows
    (1, 16, True, 3500, 0, 0),            # cut evenly
    (1, 16, True, 3500, 2000, 4)])
def test_ways_to_distribute_work(kv4, n_seqs, k, blocks, longest, window, sinks):
    hd, Hq, Hkv = 64, 4, 2
    t = H.lib_context(hd, Hq, Hkv, n_seqs * k * (k + 1 if blocks else 1))
    rng = np.random.default_rng(n_seqs + k)
    ns = _lengths(rng, n_seqs, longest) if n_seqs > 2 else [longest] + [longest // 3] * (n_seqs - 1)
    _attention_case(t, kv4, hd, Hq, Hkv, k, blocks, ns, window, sinks, 35 + n_seqs)
    t.close()


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("kv4", [True, False])
def test_absent_sequences_and_pages_outside_the_pool(impl, kv4):
    t = H.lib_context(128, 8, 2, 300, impl=impl)
    for k, blocks, ns in ((1, False, [200, -1, 64, -5]), (4, True, [-1, 100, -1, 300]), (1, False, [-1]), (16, True, [-1]), (70, False, [-1, 10])):
        _attention_case(t, kv4, 128, 8, 2, k, blocks, ns, 0, 0, 41)
        _attention_case(t, kv4, 128, 8, 2, k, blocks, ns, 90, 2, 42)

    def first_and_some(table, c):
        table[0, 0] = len(c.pools[0]); table[0, 2] = -1; table[1, 1] = 2 ** 31 - 1

    def all_of_it(table, c):
        table[:] = -7
    for k, blocks in ((1, False), (4, True), (9, False)):
        _attention_case(t, kv4, 128, 8, 2, k, blocks, [300, 190], 0, 0, 43, spoil=first_and_some)
        _attention_case(t, kv4, 128, 8, 2, k, blocks, [300, 190], 100, 80, 44, spoil=first_and_some)
        _attention_case(t, kv4, 128, 8, 2, k, blocks, [300, 190], 0, 0, 45, spoil=all_of_it)      # causal rows see nothing: zeros
    t.close()


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("kv4", [True, False])
def test_mostly_local_rows_and_the_largest_windows(impl, kv4):
    t = H.lib_context(128, 8, 2, 600, impl=impl)
    _attention_case(t, kv4, 128, 8, 2, 16, True, [0, 64], 0, 0, 46)
    _attention_case(t, kv4, 128, 8, 2, 16, True, [5], 1, 0, 47)
    _attention_case(t, kv4, 128, 8, 2, 3, True, [0, 1], 1, 1, 48)
    big = 2 ** 31 - 1
    for k, blocks, ns in ((1, False, [700, 0]), (5, True, [300]), (90, False, [70])):
        _attention_case(t, kv4, 128, 8, 2, k, blocks, ns, big, big, 49)
        _attention_case(t, kv4, 128, 8, 2, k, blocks, ns, 64, big, 50)
        _attention_case(t, kv4, 128, 8, 2, k, blocks, ns, big, 0, 51)
    t.close()


@pytest.mark.parametrize("kv4", [True, False])
@pytest.mark.parametrize("B,k,blocks,n", [(1, 1, False, 20000), (3, 1, False, 5000), (40, 1, False, 900), (1, 4, True, 9000), (1, 16, True, 4000), (2, 2, True, 3000)])
def test_a_call_gives_the_same_bits_every_time(kv4, B, k, blocks, n):
    """Partial results are merged in one order, whichever CTA does it; and a call leaves the scratch as it found it."""
    hd, Hq, Hkv = 128, 8, 2
    t = H.lib_context(hd, Hq, Hkv, 300)
    g = torch.Generator(device="cuda:0").manual_seed(4)
    width = (n + k + 63) // 64
    if kv4:
        from paper_2511_08923_b200 import kv4_page_bytes, kv4_pages
        pools = [kv4_pages(B * width, Hkv, hd) for _ in range(2)]
        for p in pools:
            x = torch.randn(B * width * 64, Hkv, hd, device="cuda:0", generator=g).to(torch.bfloat16)
            t.kv4_store(x, x, torch.arange(B * width * 64, dtype=torch.int32, device="cuda:0"), p, p)
    else:
        pools = [torch.randn(B * width, Hkv, 64, hd, device="cuda:0", generator=g).to(torch.bfloat16) for _ in range(2)]
    T = k * (k + 1) if blocks else k
    q, kl, vl = (torch.randn(r, h, hd, device="cuda:0", generator=g).to(torch.bfloat16) for r, h in ((B * T, Hq), (B * k * k, Hkv), (B * k * k, Hkv)))
    table, sl = torch.arange(B * width, dtype=torch.int32, device="cuda:0").view(B, width), _i32([n - 37 * i for i in range(B)])
    outs = [torch.zeros(B * T, Hq * hd, dtype=torch.bfloat16, device="cuda:0") for _ in range(12)]
    for o in outs:
        (t.attention_kv4 if kv4 else t.attention_window)(q, *pools, table, sl, kl if blocks else None, vl if blocks else None, o, B, k, window=0)
    t.sync()
    assert all(torch.equal(o, outs[0]) for o in outs) and outs[0].isfinite().all() and outs[0].abs().sum() > 0
    t.close()


@pytest.mark.parametrize("kv4", [True, False])
def test_lengths_beyond_the_table_are_clamped(kv4):
    t = H.lib_context(64, 4, 2, 64)
    c = H.Cache(51, kv4, 64, 2, 1, [255], garbage=False)
    q = torch.randn(1, 4, 64, device="cuda:0").to(torch.bfloat16)
    outs = [torch.zeros(1, 256, dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    for n, out in zip((255, 2 ** 31 - 1), outs):
        (t.attention_kv4 if kv4 else t.attention_window)(q, *c.pools, _i32(c.table), _i32([n]), None, None, out, 1, 1, window=0)
    t.sync()
    assert torch.equal(*outs) and outs[0].abs().sum() > 0
    t.close()


@pytest.mark.parametrize("kv4", [True, False])
def test_pools_beyond_32_bits_of_bytes(kv4):
    """Pages whose addresses lie more than 2^32 bytes into the pool."""
    hd, Hkv, n = 128, 8, 300
    t = H.lib_context(hd, 8, Hkv, 64)
    c = H.Cache(52, kv4, hd, Hkv, 1, [n], garbage=False)
    page_bytes = c.pools[0][0].numel() * c.pools[0].element_size()
    n_pages = (2 ** 32 + 2 ** 28) // page_bytes
    q = torch.randn(1, 8, hd, device="cuda:0").to(torch.bfloat16)
    outs = [torch.zeros(1, 8 * hd, dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    call = t.attention_kv4 if kv4 else t.attention_window
    call(q, *c.pools, _i32(c.table), _i32([n]), None, None, outs[0], 1, 1, window=0)
    far = n_pages - 1 - c.table.astype(np.int64)
    pools = []
    for p in c.pools:
        big = torch.empty((n_pages,) + p.shape[1:], dtype=p.dtype, device="cuda:0")
        big[torch.from_numpy(far.reshape(-1)).cuda()] = p[torch.from_numpy(c.table.reshape(-1).astype(np.int64)).cuda()]
        pools.append(big)
    call(q, *pools, _i32(far), _i32([n]), None, None, outs[1], 1, 1, window=0)
    t.sync()
    assert torch.equal(*outs) and outs[0].abs().sum() > 0
    if kv4:
        slots = _i32(far[0, 0] * 64 + np.arange(64))
        k = torch.randn(64, Hkv, hd, device="cuda:0").to(torch.bfloat16)
        a, b = torch.zeros_like(k), torch.zeros_like(k)
        t.kv4_store(k, k, slots, *pools)
        t.kv4_load(*pools, slots, a, b)
        t.sync()
        assert torch.equal(a, b) and (a.float() - k.float()).abs().max() < 0.5
    t.close()


@pytest.mark.parametrize("k,n", [(8, 500), (16, 1500), (2, 90)])
def test_without_a_window_both_agree_with_the_step_attention(k, n):
    """The same pages: through tidar_attention, through the windowed call without a window, and, as 4-bit records of the same values, through the 4-bit one."""
    hd, Hq, Hkv = 128, 8, 2
    t = H.lib_context(hd, Hq, Hkv, 300)
    four = H.Cache(61, True, hd, Hkv, k, [n], garbage=False)
    T = k * (k + 1)
    g = torch.Generator().manual_seed(3)
    q, kl, vl = (torch.randn(r, h, hd, generator=g).to(torch.bfloat16).cuda() for r, h in ((T, Hq), (k * k, Hkv), (k * k, Hkv)))
    pages = [torch.zeros(len(four.pools[0]), Hkv, 64, hd, dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    for pool, x in zip(pages, (four.K[0], four.V[0])):
        for p in range(n + k):
            pool[four.table[0, p // 64], :, p % 64] = torch.from_numpy(x[p]).to(torch.bfloat16).cuda()
    outs = [torch.zeros(T, Hq * hd, dtype=torch.bfloat16, device="cuda:0") for _ in range(3)]
    table, sl = _i32(four.table), _i32([n])
    t.attention(q, *pages, table, sl, kl, vl, outs[0], 1, k)
    t.attention_window(q, *pages, table, sl, kl, vl, outs[1], 1, k, window=0)
    t.attention_kv4(q, *four.pools, table, sl, kl, vl, outs[2], 1, k)
    t.sync()
    for o in outs[1:]:        # each is within the tolerance of the exact result: V of unit variance, so twice (2^-8 + 2^-11) of its mean magnitude and 2^-8 of the result
        assert (o.float() - outs[0].float()).abs().max() <= 2 * (2.0 ** -8 + 2.0 ** -11) * 1.5 + 2.0 ** -7 * outs[0].float().abs().max()
    t.close()


def test_a_run_of_steps_through_a_captured_graph():
    """Map, store and attend as a decoder does, captured once and replayed while lengths change on the device; drafts that are not kept give their
    pages on; each step's result is that of the rows that were stored."""
    hd, Hq, Hkv, k, B = 128, 8, 2, 4, 3
    side = torch.cuda.Stream()
    t = H.lib_context(hd, Hq, Hkv, 128, stream=side)
    T, width, n_pages = k * (k + 1), 4, 16
    rng = np.random.default_rng(71)
    from paper_2511_08923_b200 import kv4_pages
    pools = [kv4_pages(n_pages, Hkv, hd) for _ in range(2)]
    free = rng.permutation(n_pages).astype(np.int32)
    d = dict(n=_i32([0, 0, -1]), m=_i32([k] * B), held=_i32([0] * B), free=_i32(free), table=_i32(np.full((B, width), -1)), starts=_i32([0] * (B + 1)),
             slots=_i32([0] * (B * k)), counts=_i32([0] * 3))
    kv = torch.zeros(B * k, Hq + 2 * Hkv, hd, dtype=torch.bfloat16, device="cuda:0")
    q, kl, vl = (torch.zeros(r, h, hd, dtype=torch.bfloat16, device="cuda:0") for r, h in ((B * T, Hq), (B * k * k, Hkv), (B * k * k, Hkv)))
    out = torch.full((B * T, Hq * hd), 9.0, dtype=torch.bfloat16, device="cuda:0")
    torch.cuda.synchronize()

    def step():
        t.page_map(d["n"], d["m"], d["held"], d["free"], d["table"], d["held"], d["starts"], d["slots"], d["counts"], free_begin=d["counts"][:1])
        t.kv4_store(kv[:, Hq:Hq + Hkv], kv[:, Hq + Hkv:], d["slots"], *pools)
        t.attention_kv4(q, *pools, d["table"], d["n"], kl, vl, out, B, k, window=40, sinks=3)
    with torch.cuda.stream(side):
        step()                                                   # (once eagerly, with lengths that the loop sets again)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    ns = [0, 60, -1]
    d["held"].zero_(); d["counts"].zero_(); d["table"].fill_(-1)
    held, table, begin = np.zeros(B, dtype=np.int64), np.full((B, width), -1, dtype=np.int32), 0
    K, V = [[np.zeros((0, Hkv, hd))] * 3 for _ in range(2)]
    K, V = list(K), list(V)
    # sequence 1 starts with 60 positions, put in place by the same calls
    first = _rows(rng, 60, Hkv, hd) * 0.1
    first = H.bf16_round(np.nan_to_num(np.clip(first, -4, 4)))
    d["n"].copy_(_i32([-1, 0, -1])); d["m"].copy_(_i32([0, 60, 0]))
    s60 = _i32([0] * 60)
    dk = torch.from_numpy(first).to(torch.bfloat16).cuda()
    torch.cuda.synchronize()
    t.page_map(d["n"], d["m"], d["held"], d["free"], d["table"], d["held"], d["starts"], s60, d["counts"], free_begin=d["counts"][:1])
    t.kv4_store(dk, dk, s60, *pools)
    t.sync()
    table, held, _, _, counts = H.page_map(np.array([-1, 0, -1]), np.array([0, 60, 0]), held, free, 0, table, 60)
    begin = int(counts[0])
    K[1] = V[1] = H.values(*H.quantise(first))
    d["m"].copy_(_i32([k] * B))
    for turn in range(6):
        new = H.bf16_round(rng.standard_normal((B * k, Hq + 2 * Hkv, hd)))
        hq, hkl, hvl = (H.bf16_round(rng.standard_normal(tuple(x.shape))) for x in (q, kl, vl))
        for x, h in ((kv, new), (q, hq), (kl, hkl), (vl, hvl)):
            x.copy_(torch.from_numpy(h))
        d["n"].copy_(_i32(ns))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        table, held, _, slots, counts = H.page_map(np.array(ns), np.array([k] * B), held, free, begin, table, B * k)
        begin = int(counts[0])
        assert np.array_equal(d["table"].cpu().numpy(), table) and np.array_equal(d["slots"].cpu().numpy(), slots) and int(d["counts"][0]) == begin
        got = out.double().cpu().numpy()
        for i, n in enumerate(ns):
            mine = got[i * T:(i + 1) * T].reshape(T, Hq, hd)
            if n < 0:
                assert (mine == 9.0).all()
                continue
            live = sum(max(m, 0) >= 0 and a >= 0 for a, m in zip(ns[:i], [k] * i))
            rows = new[live * k:(live + 1) * k]
            k4, v4 = (H.values(*H.quantise(rows[:, a:a + Hkv])) for a in (Hq, Hq + Hkv))
            Ki, Vi = np.concatenate([K[i][:n], k4]), np.concatenate([V[i][:n], v4])
            ref, spread = H.attention(hq[i * T:(i + 1) * T], Ki, Vi, H.visible(n, k, True, 40, 3, n + k), k, hkl[i * k * k:(i + 1) * k * k], hvl[i * k * k:(i + 1) * k * k])
            assert (np.abs(mine - ref) <= H.tolerance(ref, spread)).all(), (turn, i)
            kept = 1 + (turn + i) % k
            K[i], V[i] = Ki[:n + kept], Vi[:n + kept]
            ns[i] = n + kept
    t.close()


def test_refusals_leave_everything_as_it_was():
    from paper_2511_08923_b200 import TidarError, kv4_page_bytes, kv4_pages
    from paper_2511_08923_b200.binding import tidar_attention_args
    hd, Hq, Hkv = 64, 4, 2
    t = H.lib_context(hd, Hq, Hkv, 256)
    pools = [kv4_pages(3, Hkv, hd) for _ in range(2)]
    bf = torch.bfloat16
    q, out = torch.zeros(2, Hq, hd, dtype=bf, device="cuda:0"), torch.zeros(2, Hq * hd, dtype=bf, device="cuda:0")
    loc = torch.zeros(2, Hkv, hd, dtype=bf, device="cuda:0")
    table, n = _i32([[0, 1], [2, 2]]), _i32([3, 4])
    before = t.launch_count()
    good = (q, *pools, table, n, None, None, out, 2, 1)
    bad_values = [(0, q[:1]), (0, q.float()), (0, q.cpu()), (0, q.transpose(0, 1)), (1, pools[0][:, :1]), (2, pools[1][:2]), (3, table[:1]), (3, table.long()), (4, n[:1]), (5, loc),
                  (7, out[:, :8]), (7, out.float())]
    for at, x in bad_values:
        with pytest.raises(ValueError):
            t.attention_kv4(*good[:at], x, *good[at + 1:])
    raw = dict(q=q.data_ptr(), q_stride=0, k_pages=pools[0].data_ptr(), v_pages=pools[1].data_ptr(), n_pages=3, page_table=table.data_ptr(), pages_per_seq=2, seq_len=n.data_ptr(),
               k_local=None, v_local=None, local_stride=0, out=out.data_ptr(), n_seqs=2, k=1, window=0, sinks=0)
    bad = [dict(q=None), dict(out=None), dict(seq_len=None), dict(page_table=None), dict(k_pages=None), dict(k_local=loc.data_ptr()), dict(v_local=loc.data_ptr()), dict(k=0), dict(k=-1),
           dict(n_seqs=0), dict(n_seqs=-2), dict(n_seqs=300), dict(n_seqs=2 ** 31 - 1, k=2 ** 31 - 1), dict(k=17, k_local=loc.data_ptr(), v_local=loc.data_ptr()), dict(n_pages=0),
           dict(n_pages=2 ** 25), dict(pages_per_seq=0), dict(pages_per_seq=2 ** 25), dict(pages_per_seq=1, k=65, n_seqs=1), dict(window=-1), dict(sinks=-1), dict(q_stride=100), dict(q_stride=8),
           dict(q_stride=-256), dict(local_stride=8), dict(q=q.data_ptr() + 2), dict(out=out.data_ptr() + 8), dict(seq_len=n.data_ptr() + 2)]
    for b in bad:
        for entry in (t.lib.tidar_attention_kv4, t.lib.tidar_attention_window):
            assert entry(t.ctx, C.byref(tidar_attention_args(**{**raw, **b}))) == -1, b
            assert t.lib.tidar_last_error(t.ctx)
    assert t.lib.tidar_attention_kv4(t.ctx, None) == -1 and t.lib.tidar_attention_kv4(None, C.byref(tidar_attention_args(**raw))) == -1
    k, slots = torch.zeros(4, Hkv, hd, dtype=bf, device="cuda:0"), _i32([0, 1, 2, 3])
    for args in ((k.float(), k, slots, *pools), (k, k[:3], slots, *pools), (k, k, slots.long(), *pools), (k, k, slots, pools[0][:, :, :-1], pools[1]), (k, k.transpose(0, 1), slots, *pools)):
        with pytest.raises(ValueError):
            t.kv4_store(*args)
    row = Hkv * hd
    for args in ((k.data_ptr(), row - 8, k.data_ptr(), row, slots.data_ptr(), 4, pools[0].data_ptr(), pools[1].data_ptr(), 3),
                 (k.data_ptr(), row + 4, k.data_ptr(), row, slots.data_ptr(), 4, pools[0].data_ptr(), pools[1].data_ptr(), 3),
                 (k.data_ptr() + 2, row, k.data_ptr(), row, slots.data_ptr(), 4, pools[0].data_ptr(), pools[1].data_ptr(), 3),
                 (k.data_ptr(), row, k.data_ptr(), row, slots.data_ptr(), -1, pools[0].data_ptr(), pools[1].data_ptr(), 3),
                 (k.data_ptr(), row, k.data_ptr(), row, slots.data_ptr(), 4, pools[0].data_ptr(), pools[1].data_ptr(), 0),
                 (k.data_ptr(), row, None, row, slots.data_ptr(), 4, pools[0].data_ptr(), pools[1].data_ptr(), 3)):
        assert t.lib.tidar_kv4_store(t.ctx, *args) == -1
        p, s, v, w, sl, r, a, b, m = args
        assert t.lib.tidar_kv4_load(t.ctx, a, b, m, sl, r, p, s, v, w) == -1
    t.kv4_store(k[:0], k[:0], slots[:0], *pools)                 # nothing to do is not an error
    i = [_i32([0] * 4) for _ in range(7)]
    ptr = [x.data_ptr() for x in i]
    for over in (dict(n_seqs=0), dict(n_seqs=4097), dict(width=0), dict(width=2 ** 25), dict(n_free=-1), dict(rows=-1), dict(rows=2 ** 31 - 1), dict(p=None), dict(p=ptr[0] + 1)):
        a = {**dict(n_seqs=1, width=1, n_free=1, rows=1, p=ptr[0]), **over}
        assert t.lib.tidar_page_map(t.ctx, a["p"], ptr[1], ptr[2], a["n_seqs"], ptr[3], a["n_free"], None, ptr[4], a["width"], ptr[2], ptr[5], ptr[6], a["rows"], ptr[0]) == -1, over
    with pytest.raises(ValueError):
        t.page_map(i[0], i[1], i[2], i[3], i[4], i[2], i[5], i[6], i[0])
    with pytest.raises(TidarError):
        kv4_page_bytes(96)
    t.sync()
    assert t.launch_count() == before and float(out.float().abs().sum()) == 0 and all(int(p.sum()) == 0 for p in pools)
    t.close()
