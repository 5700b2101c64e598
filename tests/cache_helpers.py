"""Plain float64 statements of the operators over a paged cache that the caller keeps, written from their documentation in tidar.h."""
import numpy as np
import torch

PAGE, GROUP = 64, 32


def bf16_round(x):
    """float64 -> nearest bf16 value (ties to even), as float64; exact in the normal range."""
    m, e = np.frexp(np.asarray(x, dtype=np.float64))
    return np.ldexp(np.rint(m * 256) / 256, e)


def bits(x):
    """bf16 values (float64) -> their 16-bit patterns."""
    return (np.asarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)


def quantise(x):
    """[..., hd] float64 -> codes [..., hd] and scale, base [..., hd / 32]."""
    x = np.where(np.isnan(x), 0.0, np.clip(x, -2.0 ** 126, 2.0 ** 126))
    g = x.reshape(x.shape[:-1] + (-1, GROUP))
    lo, hi = g.min(-1), g.max(-1)
    s = bf16_round((hi - lo) / 15)
    b = bf16_round(lo - 16 * s)
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.clip(np.rint((g - b[..., None]) / s[..., None]) - 16, 0, 15)
    return np.where(s[..., None] > 0, c, 0).astype(np.int64).reshape(x.shape), s, b


def values(c, s, b):
    g = c.reshape(c.shape[:-1] + (-1, GROUP))
    return bf16_round(b[..., None] + (16 + g) * s[..., None]).reshape(c.shape)


def records(x):
    """Pages [..., 64, hd] float64 -> their records [..., bytes] uint8."""
    c, s, b = quantise(x)
    hd = x.shape[-1]
    w = np.zeros(c.shape[:-1] + (hd // 8,), dtype=np.uint64)
    for d in range(8):
        w |= c[..., d::8].astype(np.uint64) << np.uint64(4 * (d // 2) + 16 * (d % 2))
    w = np.moveaxis(w.reshape(w.shape[:-1] + (-1, 4)), -2, -3)           # [..., group, row, word]
    codes = np.ascontiguousarray(w.astype("<u4")).view(np.uint8).reshape(c.shape[:-2] + (-1,))
    pairs = np.ascontiguousarray(np.stack([bits(s), bits(b)], -1).astype("<u2")).view(np.uint8).reshape(c.shape[:-2] + (-1,))
    return np.concatenate([codes, pairs], -1)


def page_map(n, m, held, free, begin, table, max_rows):
    """(table, held, row_start, slots, counts) as tidar_page_map leaves them."""
    table, held, width = table.copy(), held.copy(), table.shape[1]
    starts, slots, at, without = [0], [], begin, 0
    for i in range(len(n)):
        rows = max(int(m[i]), 0) if n[i] >= 0 else 0
        want = min((int(n[i]) + rows + PAGE - 1) // PAGE, width) if n[i] >= 0 else 0
        for e in range(max(held[i], 0), want):
            table[i, e] = free[at] if at < len(free) else -1
            at += 1
        held[i] = max(held[i], want)
        for j in range(rows):
            p = int(n[i]) + j
            page = table[i, p // PAGE] if p < width * PAGE else -1
            slots.append(int(page) * PAGE + p % PAGE if page >= 0 else -1)
        starts.append(starts[-1] + rows)
    without = sum(s < 0 for s in slots[:max_rows]) + max(0, len(slots) - max_rows)
    slots = (slots + [-1] * max_rows)[:max_rows]
    return table, held, np.array(starts), np.array(slots, dtype=np.int64), np.array([at, without, starts[-1]])


def visible(n, k, blocks, window, sinks, n_positions):
    """Cached positions [rows, n_positions] that the rows of a sequence of length n see."""
    bound, p = [n + j for j in range(k)], [n + j for j in range(k)]              # causal slots, then the blocks' mask slots
    if blocks:
        bound += [n + b for b in range(k) for i in range(k)]
        p += [n + b + 1 + i for b in range(k) for i in range(k)]
    t, bound, p = np.arange(n_positions)[None], np.array(bound)[:, None], np.array(p)[:, None]
    seen = t <= bound
    return seen & ((t < sinks) | (t > p - window)) if window else seen


def attention(q, K, V, vis, k, kl=None, vl=None):
    """q [T, Hq, hd]; K, V [positions, Hkv, hd]; vis [T, positions]; kl, vl [k * k, Hkv, hd].  Returns (out, mean of |v| under the weights), [T, Hq, hd].

    The second gives the bound of what rounding the weights to bf16 does: every weight is off by at most 2^-8 of itself."""
    T, Hq, hd = q.shape
    G = Hq // K.shape[1]
    if kl is not None:
        slot = np.arange(T)[:, None]
        own = (slot >= k) & (np.arange(k * k)[None] // k == (slot - k) // k)
        K, V, vis = np.concatenate([K, kl]), np.concatenate([V, vl]), np.concatenate([vis, own], 1)
    out, spread = np.zeros((T, Hq, hd)), np.zeros((T, Hq, hd))
    for h in range(Hq):
        s = np.where(vis, q[:, h] @ K[:, h // G].T / np.sqrt(hd), -np.inf)
        top = s.max(-1, keepdims=True, initial=-1e300)
        p = np.exp(s - top)
        total = p.sum(-1, keepdims=True)
        p /= np.where(total > 0, total, 1)
        out[:, h], spread[:, h] = p @ V[:, h // G], p @ np.abs(V[:, h // G])
    return out, spread


def tolerance(out, spread):
    """Element-wise: the weights' rounding to bf16 (at most 2^-8 of each, so 2^-8 of the mean of |v|), the result's own (2^-8 of it), and 2^-11 of the mean of
    |v| for the arithmetic in 32 bits: scores are sums of hd = 128 products, off by at most 128 * 2^-24 of sum |q k| / sqrt(hd), which stays below 2^5 for the
    inputs here, hence weights by 2^-12 of themselves; sums over fewer than 2^12 keys by another 2^-12."""
    return (2.0 ** -8 + 2.0 ** -11) * spread + 2.0 ** -8 * np.abs(out) + 1e-30


def lib_context(hd, Hq, Hkv, rows, k_max=16, impl=0, stream=None):
    """A library context for the stand-alone calls: its head layout, stream and scratch are what counts."""
    from dataclasses import replace
    from paper_2511_08923_b200 import Tidar, pack_weights
    from tidar_synth import CONFIGS, gen_model_weights
    sh = replace(CONFIGS["tiny"], head_dim=hd, n_q_heads=Hq, n_kv_heads=Hkv, n_layers=1, vocab=64, d_ffn=64, d_model=64)
    return Tidar(sh, pack_weights(gen_model_weights(sh), "cuda:0"), k_max=k_max, max_batch=1, max_seq_len=128, impl=impl, prefill_rows=rows, stream=stream)


class Cache:
    """Seeded pages of a batch (4 bits or bf16) in scrambled order, with garbage wherever nothing was stored, and the rows that they stand for."""

    def __init__(self, seed, kv4, hd, Hkv, k, ns, extra_pages=3, garbage=True):
        rng = np.random.default_rng(seed)
        per = [(n + k + PAGE - 1) // PAGE if n >= 0 else 0 for n in ns]
        self.width = max(max(per), 1)
        order = rng.permutation(sum(per) + extra_pages)
        self.table = np.full((len(ns), self.width), -1, dtype=np.int32)
        self.K, self.V = [], []
        shape = (sum(per) + extra_pages, Hkv, PAGE, hd)
        pools = [np.full(shape, np.nan) for _ in range(2)]
        used, at = order[:sum(per)], 0
        for i, n in enumerate(ns):
            self.table[i, :per[i]] = used[at:at + per[i]]
            at += per[i]
            for out, pool, off in ((self.K, pools[0], 0.3), (self.V, pools[1], 0.0)):
                x = bf16_round(rng.standard_normal((max(n + k, 0) if n >= 0 else 0, Hkv, hd)) + off * rng.standard_normal((Hkv, hd)))
                for p in range(len(x)):
                    pool[self.table[i, p // PAGE], :, p % PAGE] = x[p]
                out.append(values(*quantise(x)) if kv4 and len(x) else x)
        self.pools = []
        for pool in pools:
            if kv4:
                rec = records(np.nan_to_num(pool))
                if garbage:                              # slots that were never written: NaN scales, any codes
                    n_codes = PAGE * hd // 2
                    never = np.isnan(pool).any((-1,))     # [page, head, place]
                    codes = np.moveaxis(rec[..., :n_codes].reshape(shape[:2] + (hd // GROUP, PAGE, 16)), 2, 3).reshape(shape[:3] + (-1,))
                    pairs = rec[..., n_codes:].reshape(shape[:3] + (-1,))
                    codes[never] = rng.integers(0, 256, codes.shape[-1])
                    pairs[never] = 0xff
                    codes = np.moveaxis(codes.reshape(shape[:3] + (hd // GROUP, 16)), 3, 2)
                    rec = np.concatenate([codes.reshape(shape[:2] + (-1,)), pairs.reshape(shape[:2] + (-1,))], -1)
                self.pools.append(torch.from_numpy(np.ascontiguousarray(rec)).cuda())
            else:
                self.pools.append(torch.from_numpy(pool if garbage else np.nan_to_num(pool)).to(torch.bfloat16).cuda())
