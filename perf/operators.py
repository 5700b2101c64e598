"""Operators for a program that keeps its own paged cache next to the library: the page map of a batch, K and V rows held in 4 bits,
and attention over such pages or over bf16 pages within a sliding window.

A case is one call (a store is followed by the load that shows what was stored).  Sizes are spread over what the repository's
configurations do: 32/8 and 12/2 heads of 128, 4/2 heads of 64, blocks of up to 16 drafts, up to 32 k cached positions.  `run`
computes the plain form in 32 bits, or, with `own`, makes the library's calls; `exact` restates the operators in 64 bits.

Definitions.
  4-bit rows: every 32 dimensions of a head have a scale s = bf16((max - min) / 15) and a base b = bf16(min - 16 s); an element x is
  held as c = min(max(rint((x - b) / s) - 16, 0), 15) (0 where s is 0) and stands for bf16(b + (16 + c) s).  A page of a head is, for
  every group of 32 dimensions, 64 rows of 16 bytes of codes, and then 64 rows of (s, b) pairs, one for each group; element e of a row
  of codes is bits 4 (e % 8 / 2) + 16 (e % 2) of its 32-bit word e / 8.
  Attention: a sequence with n cached positions has k causal slots at n .. n + k - 1 (their K and V are in its pages) and, unless
  the call is causal, k blocks of k mask slots.  Causal slot j is at position n + j and sees positions <= n + j; slot i of block b is
  at position n + b + 1 + i and sees positions <= n + b and its own block's k local rows.  With a window w > 0 a slot at position p
  sees, of those positions, the ones below `sinks` and the ones above p - w.  Pages outside the pool are seen by no row; a row that
  sees nothing is 0; the rows of a sequence of negative length stay as they were.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
PAGE = 64
GROUP = 32
HEADS = [(32, 8, 128), (12, 2, 128), (4, 2, 64)]


def listed():
    return [
        # The tables of a small decode batch ahead of a step of up to 16 slots each: the smallest call, all latency.
        dict(name="map_decode", kind="map", seqs=32, new_lo=0, new_hi=16, n_lo=0, n_hi=4096, absent=3),
        # Many prompts at once, ragged: about 130 k rows find their places.
        dict(name="map_prompts", kind="map", seqs=509, new_lo=1, new_hi=512, n_lo=0, n_hi=2048, absent=0),
        # K and V of one step's causal slots of eight sequences, as slices of the QKV projection's output, some slots padded.
        dict(name="kv4_store_step", kind="store", hq=32, hkv=8, hd=128, rows=128, fused=True, pad=16),
        # K and V of long prompts' chunks.
        dict(name="kv4_store_prompt", kind="store", hq=32, hkv=8, hd=128, rows=20001, fused=False, pad=0),
        # One token of one request over a short 4-bit context: latency.
        dict(name="kv4_token_1k", kind="attention", bits=4, hq=32, hkv=8, hd=128, batch=1, k=1, causal=True, n_lo=1000, n_hi=1000, window=0, sinks=0, absent=0, fused=False),
        # One token each of a ragged batch: the calls that are bound by reading the cache.
        dict(name="kv4_tokens_batch", kind="attention", bits=4, hq=32, hkv=8, hd=128, batch=24, k=1, causal=True, n_lo=2999, n_hi=16001, window=0, sinks=0, absent=0, fused=True),
        # A step of 72 slots for a padded ragged batch with six query heads per KV head.
        dict(name="kv4_step_ragged", kind="attention", bits=4, hq=12, hkv=2, hd=128, batch=6, k=8, causal=False, n_lo=500, n_hi=9001, window=0, sinks=0, absent=2, fused=False),
        # A step of 272 slots over a long context: bound by arithmetic.
        dict(name="kv4_step_32k", kind="attention", bits=4, hq=32, hkv=8, hd=128, batch=1, k=16, causal=False, n_lo=32768, n_hi=32768, window=0, sinks=0, absent=0, fused=False),
        # Short blocks for a batch of long contexts of which a window and some first tokens are kept, in 4 bits.
        dict(name="kv4_step_window", kind="attention", bits=4, hq=32, hkv=8, hd=128, batch=8, k=4, causal=False, n_lo=2001, n_hi=20000, window=1024, sinks=16, absent=0, fused=False),
        # One token each on the small model with a window, bf16 pages.
        dict(name="window_tokens", kind="attention", bits=16, hq=4, hkv=2, hd=64, batch=16, k=1, causal=True, n_lo=100, n_hi=9001, window=1000, sinks=4, absent=1, fused=True),
        # The long context's step within a window of an eighth of it.
        dict(name="window_step_32k", kind="attention", bits=16, hq=32, hkv=8, hd=128, batch=1, k=16, causal=False, n_lo=32768, n_hi=32768, window=4096, sinks=4, absent=0, fused=False),
        # A chunk of a long prompt, causal, within a window.
        dict(name="window_chunk", kind="attention", bits=16, hq=32, hkv=8, hd=128, batch=1, k=1023, causal=True, n_lo=7001, n_hi=7001, window=2048, sinks=4, absent=0, fused=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["map", "store", "attention", "attention", "attention", "attention"])
    if kind == "map":
        hi = _log_int(rng, 1, 512)
        seqs = _log_int(rng, 1, min(1024, 131072 // hi))
        return dict(kind=kind, seqs=seqs, new_lo=rng.randint(0, hi), new_hi=hi, n_lo=0, n_hi=_log_int(rng, 1, 8192), absent=rng.randint(0, seqs // 4))
    hq, hkv, hd = rng.choice(HEADS)
    if kind == "store":
        rows = _log_int(rng, 1, 20000)
        return dict(kind=kind, hq=hq, hkv=hkv, hd=hd, rows=rows, fused=rng.random() < 0.5, pad=rng.randint(0, rows // 8))
    shape = rng.choice(["token", "step", "step", "chunk"])
    n_hi = _log_int(rng, 1, 32768)
    if shape == "token":
        k, causal, rows = rng.choice([1, 1, 1, rng.randint(2, 5)]), True, 1
        batch = rng.randint(1, max(1, min(32, 200000 // n_hi)))
    elif shape == "step":
        k, causal = rng.randint(1, 16), False
        rows = k * (k + 1)
        batch = rng.randint(1, max(1, min(16, 32768 // n_hi, 1088 // rows)))
    else:
        k, causal, batch = _log_int(rng, 6, 1024), True, 1
        n_hi = min(n_hi, 8000)
    window = 0 if rng.random() < 0.4 else _log_int(rng, 1, 8192)
    return dict(kind=kind, bits=rng.choice([4, 4, 16]), hq=hq, hkv=hkv, hd=hd, batch=batch, k=k, causal=causal, n_lo=int(n_hi * rng.uniform(0.0, 1.0)), n_hi=n_hi,
                window=window, sinks=rng.choice([0, 1, 4, 70]) if window else 0, absent=rng.randint(0, batch // 3), fused=rng.random() < 0.5)


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------
def _spread(lo, hi, b):
    """b numbers from lo to hi, out of order, hi first."""
    return [hi - (hi - lo) * (i * 5 % b) // max(1, b - 1) if b % 5 else hi - (hi - lo) * i // max(1, b - 1) for i in range(b)]


def _lengths(case, b):
    """Cached lengths of the batch; the last `absent` sequences are not there."""
    return [n if i < b - case["absent"] else -1 for i, n in enumerate(_spread(case["n_lo"], case["n_hi"], b))]


def _new_rows(case):
    return [m if i < case["seqs"] - case["absent"] else 0 for i, m in enumerate(_spread(case["new_lo"], case["new_hi"], case["seqs"])[::-1])]


def _rows(case):
    return case["k"] if case["causal"] else case["k"] * (case["k"] + 1)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _quantise(x):
    """Rows [..., hd] in bf16 -> (codes, scale, base), in 32 bits."""
    g = x.float().unflatten(-1, (-1, GROUP))
    lo, hi = g.amin(-1), g.amax(-1)
    fifteen = torch.full_like(lo, 15.0)
    s = ((hi - lo) / fifteen).bfloat16().float()
    b = (lo - 16 * s).bfloat16().float()
    c = (torch.round((g - b[..., None]) / s[..., None]) - 16).clamp(0, 15)
    return torch.where(s[..., None] > 0, c, torch.zeros_like(c)), s, b


def _values(c, s, b):
    return (b[..., None] + (16 + c) * s[..., None]).bfloat16().flatten(-2)


def _pack(c, s, b):
    """Codes and (scale, base) of a page [..., 64, groups, 32] as the bytes of its record."""
    w = c.transpose(-2, -3).to(torch.int64).unflatten(-1, (-1, 4, 2))     # [..., group, row, word, pair, which of it]
    at = torch.tensor([[4 * i + 16 * j for j in range(2)] for i in range(4)], device=c.device)
    w = (w << at).sum((-1, -2))
    codes = torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32).contiguous().view(torch.uint8).flatten(-3)
    pairs = torch.stack([s, b], -1).bfloat16().contiguous().view(torch.uint8).flatten(-3)
    return torch.cat([codes, pairs], -1)


def _unpack(pool, hd):
    """The values that the records [..., bytes] of a pool stand for, [..., 64, hd] in bf16."""
    n = PAGE * hd // 2
    w = pool[..., :n].contiguous().view(torch.int32).unflatten(-1, (hd // GROUP, PAGE, GROUP // 8)).transpose(-2, -3)
    at = torch.tensor([4 * i + 16 * j for i in range(4) for j in range(2)], device=pool.device, dtype=torch.int32)
    c = ((w[..., None] >> at) & 15).flatten(-2).float()
    sb = pool[..., n:].contiguous().view(torch.bfloat16).unflatten(-1, (PAGE, hd // GROUP, 2)).float()
    return _values(c, sb[..., 0], sb[..., 1])


def _normal(gen, *shape):
    return torch.randn(*shape, device=DEVICE, dtype=torch.bfloat16, generator=gen)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _handle(case):
    """The library context that such a program keeps: it gives the calls their stream and scratch."""
    from types import SimpleNamespace
    from paper_2511_08923_b200 import Tidar, pack_weights
    hq, hkv, hd = case.get("hq", 4), case.get("hkv", 2), case.get("hd", 64)
    shape = SimpleNamespace(d_model=64, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, d_ffn=64, vocab=64, tie_lm_head=False, rms_eps=1e-6, rope_theta=1e4, mask_token_id=63)

    def w(*s):
        return torch.zeros(*s, device=DEVICE, dtype=torch.bfloat16)
    layer = dict(attn_norm=w(64), ffn_norm=w(64), wq=w(hq * hd, 64), wk=w(hkv * hd, 64), wv=w(hkv * hd, 64), wo=w(64, hq * hd), w_gate=w(64, 64), w_up=w(64, 64), w_down=w(64, 64))
    packed = pack_weights(dict(embed=w(64, 64), lm_head=w(64, 64), final_norm=w(64), layers=[layer]), DEVICE)
    rows = case["batch"] * _rows(case) if case["kind"] == "attention" else 0
    return Tidar(shape, packed, k_max=16, max_batch=1, max_seq_len=128, prefill_rows=rows)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    state = dict(case=case)
    if own:
        state["lib"] = _handle(case)
    if case["kind"] == "map":
        n, m = _lengths(case, case["seqs"]), _new_rows(case)
        # a sequence may hold a page more than its length needs: what a step took and did not keep
        held = [0 if a < 0 else (a + PAGE - 1) // PAGE + (i % 3 == 1) for i, a in enumerate(n)]
        width = max(max(0, a) + b for a, b in zip(n, m)) // PAGE + 2
        need = sum((max(0, a) + b + PAGE - 1) // PAGE for a, b in zip(n, m))
        pages = torch.randperm(sum(held) + need + 8, device=DEVICE, generator=gen).to(torch.int32)
        table = torch.full((len(n), width), -1, dtype=torch.int32)
        at = 0
        for i, h in enumerate(held):
            table[i, :h] = torch.arange(at, at + h)
            at += h
        table = table.to(DEVICE)
        table = torch.where(table >= 0, pages[table.clamp(min=0).long()], table)
        rows = sum(m)
        state.update(n=_ints(n), m=_ints(m), held=_ints(held), free=pages[at:].contiguous(), begin=_ints([3]), table=table, width=width, rows=rows + 16,
                     out_table=table.clone(), out_held=torch.zeros_like(_ints(held)), starts=_ints([0] * (len(n) + 1)), slots=_ints([0] * (rows + 16)), counts=_ints([0] * 3))
        return state
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    channel = 0.5 + torch.rand(hkv, hd, device=DEVICE, generator=gen)       # K has channels that are larger than others, and off centre
    centre = torch.randn(hkv, hd, device=DEVICE, generator=gen) * 0.5
    if case["kind"] == "store":
        rows = case["rows"]
        qkv = _normal(gen, rows, hq + 2 * hkv, hd)
        k, v = qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        k.copy_((k.float() * channel + centre).bfloat16())
        if not case["fused"]:
            k, v = k.contiguous(), v.contiguous()
        n_pages = (rows + PAGE - 1) // PAGE + 3
        slots = torch.randperm(n_pages, device=DEVICE, generator=gen).repeat_interleave(PAGE)[:rows] * PAGE + torch.arange(rows, device=DEVICE) % PAGE
        slots[rows - case["pad"]:] = -1
        record = PAGE * (hd // 2 + hd // GROUP * 4)
        state.update(k=k, v=v, slots=slots.to(torch.int32), k_pages=torch.zeros(n_pages, hkv, record, dtype=torch.uint8, device=DEVICE),
                     v_pages=torch.zeros(n_pages, hkv, record, dtype=torch.uint8, device=DEVICE),
                     k_out=torch.zeros(rows, hkv, hd, dtype=torch.bfloat16, device=DEVICE), v_out=torch.zeros(rows, hkv, hd, dtype=torch.bfloat16, device=DEVICE))
        return state
    b, k, T = case["batch"], case["k"], _rows(case)
    n = _lengths(case, b)
    per = [(max(0, a) + k + PAGE - 1) // PAGE if a >= 0 else 0 for a in n]
    width, total = max(max(per), 1), sum(per)
    order = torch.randperm(total + 2, device=DEVICE, generator=gen)[:total].to(torch.int32)
    table = torch.full((b, width), -1, dtype=torch.int32, device=DEVICE)
    at = 0
    for i, p in enumerate(per):
        table[i, :p] = order[at:at + p]
        at += p

    def pool(is_k):
        out = []
        for lo in range(0, total + 2, 256):
            x = _normal(gen, min(256, total + 2 - lo), hkv, PAGE, hd)
            if is_k:
                x = (x.float() * channel[:, None] + centre[:, None]).bfloat16()
            out.append(_pack(*_quantise(x)) if case["bits"] == 4 else x)
        return torch.cat(out)
    q = _normal(gen, b * T, hq + 2 * hkv, hd)[:, :hq] if case["fused"] else _normal(gen, b * T, hq, hd)
    local = None if case["causal"] else (_normal(gen, b * k * k, hkv, hd) * channel + centre).bfloat16()
    state.update(q=q, k_pages=pool(True), v_pages=pool(False), table=table, n=_ints(n), k_local=local, v_local=None if case["causal"] else _normal(gen, b * k * k, hkv, hd),
                 out=torch.zeros(b * T, hq * hd, dtype=torch.bfloat16, device=DEVICE))
    return state


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    return {"map": _run_map, "store": _run_store, "attention": _run_attention}[state["case"]["kind"]](state)


def _run_map(s):
    if own:
        s["lib"].page_map(s["n"], s["m"], s["held"], s["free"], s["out_table"], s["out_held"], s["starts"], s["slots"], s["counts"], free_begin=s["begin"])
        return dict(table=s["out_table"], held=s["out_held"], starts=s["starts"], slots=s["slots"], counts=s["counts"])
    n, m, held, width = s["n"].clamp(min=0), s["m"].clamp(min=0) * (s["n"] >= 0), s["held"], s["width"]
    want = ((n + m + PAGE - 1) // PAGE).clamp(max=width) * (s["n"] >= 0)
    take = (want - held).clamp(min=0)
    first = s["begin"] + take.cumsum(0) - take
    entry = torch.arange(width, device=DEVICE)[None]
    at = (first[:, None] + entry - held[:, None]).long()
    fresh = (entry >= held[:, None]) & (entry < want[:, None])
    table = torch.where(fresh, torch.where(at < len(s["free"]), s["free"][at.clamp(0, len(s["free"]) - 1)], -1), s["table"])
    starts = torch.cat([torch.zeros_like(m[:1]), m.cumsum(0).to(torch.int32)])
    row = torch.arange(s["rows"], device=DEVICE)
    seq = torch.searchsorted(starts[1:].contiguous(), row.to(torch.int32), right=True).clamp(max=len(n) - 1)
    pos = n[seq] + row - starts[seq]
    page = table[seq, (pos // PAGE).clamp(0, width - 1)]
    live = row < starts[-1]
    good = live & (pos < width * PAGE) & (page >= 0)
    counts = torch.stack([s["begin"][0] + take.sum(), (live & ~good).sum(), starts[-1]])
    return dict(table=table.to(torch.int32), held=torch.maximum(held, want).to(torch.int32), starts=starts.to(torch.int32),
                slots=torch.where(good, page * PAGE + pos % PAGE, -1).to(torch.int32), counts=counts.to(torch.int32))


def _run_store(s):
    if own:
        s["lib"].kv4_store(s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"])
        s["lib"].kv4_load(s["k_pages"], s["v_pages"], s["slots"], s["k_out"], s["v_out"])
        return dict(k=s["k_out"], v=s["v_out"])
    kept = (s["slots"] >= 0)[:, None, None]
    return dict(k=torch.where(kept, _values(*_quantise(s["k"])), s["k_out"]), v=torch.where(kept, _values(*_quantise(s["v"])), s["v_out"]))


def _run_attention(s):
    case = s["case"]
    if own:
        call = s["lib"].attention_kv4 if case["bits"] == 4 else s["lib"].attention_window
        call(s["q"], s["k_pages"], s["v_pages"], s["table"], s["n"], s["k_local"], s["v_local"], s["out"], case["batch"], case["k"], window=case["window"], sinks=case["sinks"])
        return s["out"]
    b, k, T, hq, hkv, hd = case["batch"], case["k"], _rows(case), case["hq"], case["hkv"], case["hd"]
    n, table = s["n"].long(), s["table"].long()
    there = (table >= 0) & (table < len(s["k_pages"]))

    def keys(pool, local):
        x = pool[table.clamp(0, len(pool) - 1)]                                          # [b, page, head, ...]
        x = (_unpack(x, hd) if case["bits"] == 4 else x).float().transpose(2, 3).flatten(1, 2)   # [b, position, head, hd]
        return (x if local is None else torch.cat([x, local.float().view(b, k * k, hkv, hd)], 1)).transpose(1, 2)
    kk, vv = keys(s["k_pages"], s["k_local"]), keys(s["v_pages"], s["v_local"])
    slot = torch.arange(T, device=DEVICE)
    block = torch.where(slot < k, slot, (slot - k) // k)                                 # a slot of block b sees what causal slot b sees
    ahead = torch.where(slot < k, slot, block + 1 + (slot - k) % k)                      # its position, from n on
    t = torch.arange(table.shape[1] * PAGE, device=DEVICE)
    seen = (t <= (n[:, None] + block)[..., None]) & there.repeat_interleave(PAGE, 1)[:, None]
    if case["window"]:
        seen &= (t < case["sinks"]) | (t > (n[:, None] + ahead)[..., None] - case["window"])
    if not case["causal"]:
        own_block = (torch.arange(k * k, device=DEVICE) // k == block[:, None]) & (slot >= k)[:, None]
        seen = torch.cat([seen, own_block.expand(b, -1, -1)], -1)
    q = s["q"].float().view(b, T, hkv, hq // hkv, hd).permute(0, 2, 3, 1, 4)            # [b, head, group, slot, hd]
    vv = torch.where(seen.any(1)[:, None, :, None], vv, torch.zeros((), device=DEVICE))
    score = (q.flatten(2, 3) @ kk.transpose(-1, -2)).view(b, hkv, hq // hkv, T, -1) / math.sqrt(hd)
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    p = (p / torch.where(total > 0, total, torch.ones_like(total))).flatten(2, 3)
    out = (p @ vv).view(b, hkv, hq // hkv, T, hd).permute(0, 3, 1, 2, 4).reshape(b, T, hq * hd).bfloat16()
    return torch.where((n >= 0)[:, None, None], out, s["out"].view(b, T, -1)).view(b * T, -1)


# ---------------------------------------------------------------------------
# the same in 64 bits, sequence by sequence
# ---------------------------------------------------------------------------
def _bf16(x):
    """Nearest value of eight significant bits, ties to even."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 256) / 256, e)


def _stored(x):
    """What rows of [..., hd] stand for once they are held in 4 bits."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for lo in range(0, x.shape[-1], GROUP):
        g = x[..., lo:lo + GROUP].double()
        s = _bf16((g.amax(-1, keepdim=True) - g.amin(-1, keepdim=True)) / torch.full((), 15.0, dtype=torch.float64, device=x.device))
        b = _bf16(g.amin(-1, keepdim=True) - 16 * s)
        c = torch.where(s > 0, torch.round((g - b) / torch.where(s > 0, s, torch.ones_like(s))) - 16, torch.zeros_like(g))
        out[..., lo:lo + GROUP] = _bf16(b + (16 + c.clamp(0, 15)) * s)
    return out


def _read(pool, page, hd):
    """The rows [head, 64, hd] of one page of 4-bit records."""
    rec = pool[page]
    raw = rec[:, :PAGE * hd // 2].reshape(-1, hd // GROUP, PAGE, GROUP // 8, 4).permute(0, 2, 1, 3, 4).reshape(-1, PAGE, hd // 8, 4).long()
    word = raw[..., 0] + (raw[..., 1] << 8) + (raw[..., 2] << 16) + (raw[..., 3] << 24)
    code = torch.stack([(word >> (4 * (d // 2) + 16 * (d % 2))) & 15 for d in range(8)], -1).flatten(-2).double()
    sb = rec[:, PAGE * hd // 2:].contiguous().view(torch.bfloat16).reshape(-1, PAGE, hd // GROUP, 2).double().repeat_interleave(GROUP, 2)
    return _bf16(sb[..., 1] + (16 + code) * sb[..., 0])


def exact(case, seed):
    if case["kind"] == "map":
        return None                                          # whole numbers
    s = prepare(case, seed)
    if case["kind"] == "store":
        live = (s["slots"] >= 0).double()[:, None, None]
        return dict(k=_stored(s["k"]) * live, v=_stored(s["v"]) * live)
    b, k, T, hq, hkv, hd = case["batch"], case["k"], _rows(case), case["hq"], case["hkv"], case["hd"]
    out = torch.zeros(b * T, hq, hd, dtype=torch.float64, device=DEVICE)
    for i, n in enumerate(s["n"].tolist()):
        if n < 0:
            continue
        pages = s["table"][i].tolist()[:(n + k + PAGE - 1) // PAGE]
        K, V = (torch.cat([_read(pool, p, hd) if case["bits"] == 4 else pool[p].double() for p in pages], 1) for pool in (s["k_pages"], s["v_pages"]))
        t = torch.arange(K.shape[1], device=DEVICE)

        def attend(rows, bound, p, keys=None, values=None):
            """rows [r]: slots that see positions <= bound [r], being at positions p [r], and local keys [head, key, hd]."""
            vis = t[None] <= bound[:, None]
            if case["window"] > 0:
                vis &= (t[None] < case["sinks"]) | (p[:, None] - t[None] < case["window"])
            for h in range(hkv):
                q = s["q"][i * T + rows, h * (hq // hkv):(h + 1) * (hq // hkv)].double()
                sc = torch.einsum("rgd,td->rgt", q, K[h]).masked_fill(~vis[:, None], -math.inf)
                v = V[h]
                if keys is not None:
                    sc, v = torch.cat([sc, torch.einsum("rgd,td->rgt", q, keys[h])], -1), torch.cat([v, values[h]])
                out[i * T + rows, h * (hq // hkv):(h + 1) * (hq // hkv)] = torch.softmax(sc / hd ** 0.5, -1) @ v
        for lo in range(0, k, 128):
            j = torch.arange(lo, min(lo + 128, k), device=DEVICE)
            attend(j, n + j, n + j)
        for blk in range(0 if case["causal"] else k):
            j = torch.arange(k, device=DEVICE)
            local = slice((i * k + blk) * k, (i * k + blk + 1) * k)
            attend(k + blk * k + j, torch.full_like(j, n + blk), n + blk + 1 + j, s["k_local"][local].double().transpose(0, 1), s["v_local"][local].double().transpose(0, 1))
    return out.view(b * T, hq * hd)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    if case["kind"] == "map":
        n, m = _lengths(case, case["seqs"]), _new_rows(case)
        entries = sum((a + r + PAGE - 1) // PAGE - a // PAGE for a, r in zip(n, m) if a >= 0)
        return {"bytes": 4 * (sum(m) + 3 * entries + 5 * len(n)), "flops": sum(m)}
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    row4 = hkv * (hd // 2 + hd // GROUP * 4)                 # bytes of K or V of a position in 4 bits
    if case["kind"] == "store":
        return {"bytes": 2 * case["rows"] * (2 * 2 * hkv * hd + 2 * row4), "flops": 8 * case["rows"] * hkv * hd}
    row, k, w = row4 if case["bits"] == 4 else 2 * hkv * hd, case["k"], case["window"]
    total = flops = 0
    for n in _lengths(case, case["batch"]):
        if n < 0:
            continue

        def seen(bound, p):                                  # positions <= bound that a slot at position p sees
            return bound + 1 if w == 0 else min(bound + 1, case["sinks"]) + max(0, bound + 1 - max(case["sinks"], p - w + 1, 0))
        pairs = sum(seen(n + j, n + j) for j in range(k))
        if not case["causal"]:
            pairs += sum(seen(n + b, n + b + 1 + i) + k for b in range(k) for i in range(k))
            total += 2 * 2 * k * k * hkv * hd
        first = max(0, n - w + 1) if w else 0                # the first slot's window reaches furthest back
        total += 2 * row * (n + k - max(0, first - case["sinks"])) + 4 * _rows(case) * hq * hd
        flops += 4 * hq * hd * pairs
    return {"bytes": total, "flops": flops}
