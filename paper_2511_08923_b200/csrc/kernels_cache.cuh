// A paged cache that the caller keeps: page map of a batch, K and V rows held in 4 bits, and the plain attention over such pages or bf16
// pages with a sliding window.  (The kernels that read them fast: attn_few.cuh, attn_tc.cuh.)
#pragma once
#include "common.cuh"
#include "sm100_ptx.cuh"

// ---- rows in 4 bits --------------------------------------------------------------------
// Every 32 dimensions of a head (a group) have a scale s = bf16((max - min) / 15) and a base b = bf16(min - 16 s).  An element is held as
// a code c in 0 .. 15 and stands for bf16(b + (16 + c) s).  The base lies 16 scales below the minimum because 16 + c is a bf16 number whose
// mantissa holds c: (code << 3) | 0x4180 is that number, so a reader gets from codes to values with one shift, one logical operation and one
// packed FMA for two of them, and no subtraction.  (Rounding such a base costs at most 2^-9 of about 24 s for centred groups: 0.05 s.)
// A page of a head is one record: for each group 64 rows of 16 bytes of codes, then 64 rows of (s, b) pairs.  Element e of a group is bits
// 4 (e % 8 / 2) + 16 (e % 2) of the row's 32-bit word e / 8, so that a shift brings two neighbours to the places of a pair of bf16 numbers; and
// lanes that take a row each read 16 bytes next to one another.
namespace kv4 {
constexpr int PAGE = 64, GROUP = 32;
__host__ __device__ constexpr int code_bytes(int hd) { return PAGE * hd / 2; }
__host__ __device__ constexpr int record_bytes(int hd) { return PAGE * (hd / 2 + hd / GROUP * 4); }
__host__ __device__ constexpr int word_at(int place, int w) { return (w / 4 * PAGE + place) * 16 + w % 4 * 4; }      // of dimensions 8 w .. 8 w + 7
constexpr float LARGEST = 8.507059173023462e37f;      // 2^126: twice that, and a base 16 scales away (-1.57 * 2^127), are still finite; their difference need not be (see codes8)

// Four pairs of values (dimensions 8 w .. 8 w + 7) of word `w`; ss = (s, s), bb = (b, b).
__device__ __forceinline__ uint32_t pair_of(uint32_t shifted, uint32_t ss, uint32_t bb) {
  uint32_t v, r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(v) : "r"(shifted), "r"(0x00780078u), "r"(0x41804180u));      // (shifted & mask) | 16: written in C it became two instructions
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(v), "r"(ss), "r"(bb));
  return r;
}
__device__ __forceinline__ void values8(uint32_t w, uint32_t ss, uint32_t bb, uint32_t (&out)[4]) {
  out[0] = pair_of(w << 3, ss, bb); out[1] = pair_of(w >> 1, ss, bb); out[2] = pair_of(w >> 5, ss, bb); out[3] = pair_of(w >> 9, ss, bb);
}
__device__ __forceinline__ uint32_t low_twice(uint32_t sb) { return __byte_perm(sb, 0, 0x1010); }
__device__ __forceinline__ uint32_t high_twice(uint32_t sb) { return __byte_perm(sb, 0, 0x3232); }
}  // namespace kv4

// Blocks of kv4_store_kernel / kv4_load_kernel: threads take eight dimensions each, x along a row (several turns where it has more than KV4_THREADS), y rows.
constexpr int KV4_THREADS = 256;
__host__ inline dim3 kv4_block(int heads, int hd) {
  const int per_row = heads * hd / 8;
  return per_row < KV4_THREADS ? dim3(per_row, KV4_THREADS / per_row) : dim3(KV4_THREADS, 1);
}

namespace kv4 {
// d / 15, correctly rounded in the same way (see below).
__device__ __forceinline__ float fifteenth(float d) {
  constexpr float R = 1.f / 15.f;
  const float q = d * R;
  return d > 1e-30f ? fmaf(fmaf(-q, 15.f, d), R, q) : __fdiv_rn(d, 15.f);
}
// The codes of eight elements as a word.  The quotient is corrected once by its exact remainder, which makes it the correctly rounded one (Markstein: the
// reciprocal is correctly rounded and s, a bf16 number, not the largest of its binade), so that ties, of which numbers of eight bits have many, are ties.
// Nothing else must be one.  A distance y = x - b > 0 that is off a border between two codes is so by a unit of its last place at least, which is more than
// half a unit of the quotient's.  But where x - b does not fit 32 bits, rounding it can bring it onto a border.  With s in [2^e, 2^(e+1)) borders are multiples
// of 2^(e-8) (b, near -16 s or further out wherever there is an x that small, and s have eight bits), and y is below 2^(e+6), so that this takes an x within
// 2^(e-18) of a border at 0.  A tie there goes to the even one of its neighbours: where that is the upper one distances are rounded down, otherwise up, and
// what lands on the border goes the way that it should have gone without.
__device__ __forceinline__ uint32_t codes8(const float (&x)[8], float s, float b) {
  using namespace sm100;
  constexpr float MAGIC = 12582912.f;                  // 1.5 * 2^23: adding it rounds to an integer, ties to even, which are then the low bits
  const float inv = __frcp_rn(s);
  float r[8];                                          // the quotients, rounded, + MAGIC
  // rounded up, a distance is the negative of its negative rounded down: all signs are `up`'s
  const uint32_t up = ~__float_as_uint(fmaf(-b, inv, -0.5f) + MAGIC) << 31;       // (the integer below a border at 0 is even)
  auto sign = [&](float v) { return __uint_as_float(__float_as_uint(v) ^ up); };
  const float one = sign(1.f), nb = sign(-b), ss = sign(s), si = sign(inv);
#pragma unroll
  for (int e = 0; e < 8; e += 2) {                     // (in pairs: 42.5 us one by one)
    const f32x2 y = fma2_down(pack2(x[e], x[e + 1]), pack2(one, one), pack2(nb, nb)), q = mul2(y, pack2(si, si));
    unpack2(add2(fma2(fma2(q, pack2(-ss, -ss), y), pack2(si, si), q), pack2(MAGIC, MAGIC)), r[e], r[e + 1]);
  }
  if (!(s > 1e-30f && s < 1e30f)) {                    // where remainders or the reciprocal leave the range of normal numbers; and a scale of 0, which gives code 0
    const float part = s < 1.f ? 1.f : 0.25f;          // (x - b reaches 2^128.05: of large numbers quarters are divided, which changes no quotient)
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (s > 0.f ? fminf(fmaxf(__fdiv_rn(__fmaf_rd(x[e], one * part, nb * part), ss * part), 0.f), 100.f) : 0.f) + MAGIC;
  }
  // as integers r is 0x4b400000 and 16 .. 31; the multiples of 0x4b400010 that are summed with the codes are taken off at the end (modulo 2^32)
  uint32_t w = 0, extra = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t place = 1u << (4 * (e / 2) + 16 * (e % 2));
    w += (uint32_t)min(max(__float_as_int(r[e]), 0x4b400010), 0x4b40001f) * place;
    extra += 0x4b400010u * place;
  }
  return w - extra;
}
}  // namespace kv4

// Rows of K and V to the slots (64 page + place) that the page map gave them; a slot outside the pool is skipped.  Four threads share a group of 32
// dimensions, eight each; a thread takes the same place of K and V, so that two loads are on their way at once.  Instructions bound it, most of
// them for the codes (20001 rows of 8 heads of 128: 40 us, 108 MB; 44 with the five blocks per SM that fit without asking for six, which spill 20 bytes a thread).
template <int HD>
__global__ void __launch_bounds__(KV4_THREADS, 6) kv4_store_kernel(const bf16 *k, long long k_stride, const bf16 *v, long long v_stride, const int32_t *slots,
                                                                int n_rows, int heads, uint8_t *k_pages, uint8_t *v_pages, int n_pages) {
  constexpr int PER_HEAD = HD / 8;
  const int per_row = heads * PER_HEAD;                // (a multiple of eight: the four threads of a group lie in one warp, full or not)
  const long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  const bool there = row < n_rows;
  pdl_trigger();
  pdl_wait();
  const int slot = there ? slots[row] : -1;
  const bool live = slot >= 0 && slot / kv4::PAGE < n_pages;
  const int place = slot & (kv4::PAGE - 1);
  const int first_lane = (threadIdx.y * blockDim.x + threadIdx.x) & ~31, lanes = blockDim.x * blockDim.y - first_lane;
  const unsigned warp_lanes = lanes >= 32 ? 0xffffffffu : (1u << lanes) - 1;      // (the block's last warp may have fewer)
  for (int at0 = 0; at0 < per_row; at0 += blockDim.x) {      // (all threads take every turn: the exchange below is of whole warps)
    const bool has = there && at0 + (int)threadIdx.x < per_row;
    const int at = has ? at0 + threadIdx.x : 0, head = at / PER_HEAD, part = at % PER_HEAD;
    uint4 raw[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (has) {
      raw[0] = *reinterpret_cast<const uint4 *>(k + row * k_stride + at * 8);
      raw[1] = *reinterpret_cast<const uint4 *>(v + row * v_stride + at * 8);
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      uint32_t w[4] = {raw[which].x, raw[which].y, raw[which].z, raw[which].w};
      // what is held is finite: magnitudes above 2^126 (0x7e80) become that, NaN becomes 0
      uint32_t large = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) large |= (w[e] & 0x7fff7fffu) + 0x017f017fu;
      if (large & 0x80008000u) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162 *>(&w[e]));
          const __nv_bfloat162 h = __floats2bfloat162_rn(f.x != f.x ? 0.f : fminf(fmaxf(f.x, -kv4::LARGEST), kv4::LARGEST), f.y != f.y ? 0.f : fminf(fmaxf(f.y, -kv4::LARGEST), kv4::LARGEST));
          w[e] = *reinterpret_cast<const uint32_t *>(&h);
        }
      }
      __nv_bfloat162 lo2 = *reinterpret_cast<__nv_bfloat162 *>(&w[0]), hi2 = lo2;
      float x[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const __nv_bfloat162 h = *reinterpret_cast<__nv_bfloat162 *>(&w[e]);
        lo2 = __hmin2(lo2, h); hi2 = __hmax2(hi2, h);
        const float2 f = __bfloat1622float2(h);
        x[2 * e] = f.x; x[2 * e + 1] = f.y;
      }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) { lo2 = __hmin2(lo2, __shfl_xor_sync(warp_lanes, lo2, o)); hi2 = __hmax2(hi2, __shfl_xor_sync(warp_lanes, hi2, o)); }
      const float lo = fminf(__low2float(lo2), __high2float(lo2)), hi = fmaxf(__low2float(hi2), __high2float(hi2));
      const bf16 s16 = __float2bfloat16_rn(kv4::fifteenth(hi - lo));
      const float s = __bfloat162float(s16);
      const bf16 b16 = __float2bfloat16_rn(lo - 16.f * s);
      const uint32_t code = kv4::codes8(x, s, __bfloat162float(b16));
      if (has && live) {
        uint8_t *rec = (which ? v_pages : k_pages) + ((size_t)(slot / kv4::PAGE) * heads + head) * kv4::record_bytes(HD);
        *reinterpret_cast<uint32_t *>(rec + kv4::word_at(place, part)) = code;
        if (part % 4 == 0)
          *reinterpret_cast<uint32_t *>(rec + kv4::code_bytes(HD) + (place * (HD / kv4::GROUP) + part / 4) * 4) = (uint32_t)__bfloat16_as_ushort(s16) | (uint32_t)__bfloat16_as_ushort(b16) << 16;
      }
    }
  }
}

// (No __restrict__: rows, slots and pages may be the previous kernel's output, which ends after this one has begun.)
// The values at the listed slots as rows of K and V; a row whose slot is outside the pool is left as it is.  20001 rows of 8 heads of 128: 23.4 us, 108 MB, 1.4 of
// the time that memory needs for them.  A thread waits for its slot and then for its codes, and issue slots are half full (52 %).
template <int HD>
__global__ void __launch_bounds__(KV4_THREADS) kv4_load_kernel(const uint8_t *k_pages, const uint8_t *v_pages, int n_pages, const int32_t *slots, int n_rows,
                                                               int heads, bf16 *k, long long k_stride, bf16 *v, long long v_stride) {
  constexpr int PER_HEAD = HD / 8;
  const long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  pdl_trigger();
  pdl_wait();
  if (row >= n_rows) return;
  const int slot = slots[row];
  if (slot < 0 || slot / kv4::PAGE >= n_pages) return;
  const int place = slot & (kv4::PAGE - 1);
  for (int at = threadIdx.x; at < heads * PER_HEAD; at += blockDim.x) {
    const int head = at / PER_HEAD, part = at % PER_HEAD;
    const size_t rec = ((size_t)(slot / kv4::PAGE) * heads + head) * kv4::record_bytes(HD);
    const size_t code = rec + kv4::word_at(place, part), pair = rec + kv4::code_bytes(HD) + (place * (HD / kv4::GROUP) + part / 4) * 4;
    const uint32_t wk = *reinterpret_cast<const uint32_t *>(k_pages + code), wv = *reinterpret_cast<const uint32_t *>(v_pages + code);
    const uint32_t pk = *reinterpret_cast<const uint32_t *>(k_pages + pair), pv = *reinterpret_cast<const uint32_t *>(v_pages + pair);
    uint32_t o[4];
    kv4::values8(wk, kv4::low_twice(pk), kv4::high_twice(pk), o);
    *reinterpret_cast<uint4 *>(k + row * k_stride + at * 8) = make_uint4(o[0], o[1], o[2], o[3]);
    kv4::values8(wv, kv4::low_twice(pv), kv4::high_twice(pv), o);
    *reinterpret_cast<uint4 *>(v + row * v_stride + at * 8) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// ---- page map ------------------------------------------------------------------------------
struct PageMapArgs {
  int n_seqs, n_free, width, max_rows;
  const int32_t *seq_len, *n_new, *held, *free_pages, *free_begin;    // (free_begin may be null: 0)
  int32_t *table, *held_out, *row_start, *slots, *counts;
  int32_t *scratch;                     // [2], zero between calls: CTAs that are done, rows without a slot
};
constexpr int MAP_THREADS = 512, MAP_ROWS = 2048, MAP_MAX_SEQS = 4096;

// Every CTA works out all sequences' first row and first fresh page (one scan over the lengths: cheaper than a second kernel that waits for the
// first) and then fills its share of the slots and of the table.  The table entries that a sequence holds are only read and the ones behind them
// only written, a fresh page is taken from the free list wherever it is needed, so the CTAs need nothing from one another; what may be
// overwritten in place (held, the counters) is written by the CTA that finishes last.  Sums saturate.
// Bound by latency: two dependent loads, a scan, a search.
__global__ void __launch_bounds__(MAP_THREADS) page_map_kernel(const PageMapArgs a) {
  extern __shared__ int32_t map_smem[];
  int32_t *first_row = map_smem, *first_page = map_smem + a.n_seqs + 1;       // [n_seqs + 1] each
  __shared__ int warp_rows[MAP_THREADS / 32], warp_pages[MAP_THREADS / 32];
  __shared__ int missing, last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_trigger();
  pdl_wait();
  auto plus = [](int x, int y) { return (int)min((unsigned)x + (unsigned)y, 0x7fffffffu); };
  struct Seq { int n, m, held, want; };
  auto seq_of = [&](int i) {
    Seq s;
    s.n = a.seq_len[i];
    s.m = s.n < 0 ? 0 : max(a.n_new[i], 0);
    s.held = min(max(a.held[i], 0), a.width);
    s.want = s.n < 0 ? 0 : (int)min(((long long)s.n + s.m + 63) / 64, (long long)a.width);
    return s;
  };
  const int per = (a.n_seqs + MAP_THREADS - 1) / MAP_THREADS, i0 = min(tid * per, a.n_seqs), i1 = min(i0 + per, a.n_seqs);
  int rows = 0, pages = 0;
  for (int i = i0; i < i1; ++i) { const Seq s = seq_of(i); rows = plus(rows, s.m); pages = plus(pages, max(s.want - s.held, 0)); }
  int sum_rows = rows, sum_pages = pages;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, sum_rows, o), y = __shfl_up_sync(0xffffffffu, sum_pages, o);
    if (lane >= o) { sum_rows = plus(sum_rows, x); sum_pages = plus(sum_pages, y); }
  }
  if (lane == 31) { warp_rows[warp] = sum_rows; warp_pages[warp] = sum_pages; }
  if (tid == 0) missing = 0;
  __syncthreads();
  int at_row = __shfl_up_sync(0xffffffffu, sum_rows, 1), at_page = __shfl_up_sync(0xffffffffu, sum_pages, 1);
  if (lane == 0) at_row = at_page = 0;
  for (int w = 0; w < warp; ++w) { at_row = plus(at_row, warp_rows[w]); at_page = plus(at_page, warp_pages[w]); }
  const int begin = a.free_begin ? max(*a.free_begin, 0) : 0;
  at_page = plus(at_page, begin);
  for (int i = i0; i < i1; ++i) {
    const Seq s = seq_of(i);
    first_row[i] = at_row; first_page[i] = at_page;
    at_row = plus(at_row, s.m); at_page = plus(at_page, max(s.want - s.held, 0));
  }
  if (i0 < i1 && i1 == a.n_seqs) { first_row[a.n_seqs] = at_row; first_page[a.n_seqs] = at_page; }
  __syncthreads();
  const int total = first_row[a.n_seqs];
  auto fresh = [&](int at) { return at < a.n_free ? a.free_pages[at] : -1; };        // (saturated sums lie behind any list)
  // table entries: a warp per sequence
  for (int i = blockIdx.x * (MAP_THREADS / 32) + warp; i < a.n_seqs; i += gridDim.x * (MAP_THREADS / 32)) {
    const Seq s = seq_of(i);
    for (int e = s.held + lane; e < s.want; e += 32) a.table[(size_t)i * a.width + e] = fresh(plus(first_page[i], e - s.held));
    if (lane == 0) a.row_start[i] = first_row[i];
  }
  // slots
  int none = 0;
  for (int r = blockIdx.x * MAP_ROWS + tid; r < min((blockIdx.x + 1) * MAP_ROWS, a.max_rows); r += MAP_THREADS) {
    int slot = -1;
    if (r < total) {
      int lo = 0, hi = a.n_seqs;                       // the last sequence whose first row is at most r
      while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (first_row[mid] <= r) lo = mid; else hi = mid; }
      const long long pos = (long long)a.seq_len[lo] + (r - first_row[lo]);
      const int held = min(max(a.held[lo], 0), a.width);
      if (pos < (long long)a.width * 64) {
        const int e = (int)(pos >> 6);
        const int page = e < held ? a.table[(size_t)lo * a.width + e] : fresh(plus(first_page[lo], e - held));
        if (page >= 0 && page < (1 << 25)) slot = page * 64 + (int)(pos & 63);
      }
      none += slot < 0;
    }
    a.slots[r] = slot;
  }
  none = __reduce_add_sync(0xffffffffu, none);
  if (lane == 0 && none) atomicAdd(&missing, none);
  __threadfence();
  __syncthreads();
  if (tid == 0) {
    if (missing) atomicAdd(&a.scratch[1], missing);
    __threadfence();
    last = atomicAdd(&a.scratch[0], 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  // every CTA has read what may be overwritten in place
  for (int i = tid; i < a.n_seqs; i += MAP_THREADS) a.held_out[i] = max(a.held[i], seq_of(i).want);
  if (tid == 0) {
    __threadfence();
    const int without = *reinterpret_cast<volatile int32_t *>(&a.scratch[1]);
    a.row_start[a.n_seqs] = total;
    a.counts[0] = first_page[a.n_seqs];
    a.counts[1] = plus(without, max(total - a.max_rows, 0));
    a.counts[2] = total;
    a.scratch[0] = 0; a.scratch[1] = 0;
  }
}

// ---- what a row of a windowed call sees -----------------------------------------------------
// The slots of a step (blocks = 1: k causal slots, then k blocks of k mask slots) or k causal slots alone.  A row sees the cached positions t < nvis with
// t < sinks or t >= low, and local rows [loc0, loc0 + nloc).  Its sequence is absent (seq_len < 0): n < 0.
struct WindowRows {
  const int32_t *seq_len; int k, blocks, n_max, window, sinks;
  __host__ __device__ int rows() const { return blocks ? k * (k + 1) : k; }
};
struct WindowKeys { int n, nvis, low, loc0, nloc, seq; };
__device__ __forceinline__ WindowKeys window_keys(const WindowRows &w, int r) {
  const int T = w.rows(), s = r / T, slot = r - s * T;
  WindowKeys o{};
  o.seq = s;
  o.n = min(w.seq_len[s], w.n_max);
  if (o.n < 0) return o;
  int pos;
  if (slot < w.k) { o.nvis = o.n + slot + 1; pos = o.n + slot; }
  else {
    const int b = (slot - w.k) / w.k;
    o.nvis = o.n + b + 1; o.loc0 = s * w.k * w.k + b * w.k; o.nloc = w.k;
    pos = o.n + b + 1 + (slot - w.k - b * w.k);
  }
  o.low = w.window > 0 ? max(pos - w.window + 1, 0) : 0;
  return o;
}

// What the attention kernels over a caller's pages are given.
struct CacheArgs {
  const bf16 *q; long long q_stride;
  const void *k_pages, *v_pages; int n_pages;
  const int32_t *table; int width;
  const bf16 *k_local, *v_local; long long local_stride;
  bf16 *out;
  int Hq, Hkv;
  WindowRows rows;
};

// One warp per (row, query head), 32 keys at a time, fp32 throughout: impl 1.
template <int HD, bool KV4>
__global__ void __launch_bounds__(32) attn_cache_replay_kernel(const CacheArgs a, float scale) {
  constexpr int DPL = HD / 32;
  __shared__ float qs[HD];
  __shared__ float vs[32][HD + 1];
  const int r = blockIdx.x, h = blockIdx.y, lane = threadIdx.x, kvh = h / (a.Hq / a.Hkv);
  const WindowKeys w = window_keys(a.rows, r);
  if (w.n < 0) return;
  const bf16 *q = a.q + r * a.q_stride + h * HD;
  for (int c = lane; c < HD; c += 32) qs[c] = __bfloat162float(q[c]) * scale;
  __syncwarp();
  float mx = -INFINITY, den = 0.f, acc[DPL] = {};
  // keys in the order: sinks, window, local rows
  const int n_sink = min(a.rows.window > 0 ? a.rows.sinks : 0, w.nvis), low = max(w.low, n_sink), n_window = max(w.nvis - low, 0), total = n_sink + n_window + w.nloc;
  for (int t0 = 0; t0 < total; t0 += 32) {
    const int t = t0 + lane;
    float sc = -INFINITY;
    bool live = false;
    auto row_of = [&](const bf16 *k, const bf16 *v) {
      float dot = 0.f;
      for (int c = 0; c < HD; ++c) { dot = fmaf(__bfloat162float(k[c]), qs[c], dot); vs[lane][c] = __bfloat162float(v[c]); }
      sc = dot; live = true;
    };
    if (t < n_sink + n_window) {
      const int pos = t < n_sink ? t : low + (t - n_sink);
      const int page = a.table[(size_t)w.seq * a.width + pos / 64];
      if ((unsigned)page < (unsigned)a.n_pages) {        // (a page outside the pool is seen by no row)
        const size_t head = (size_t)page * a.Hkv + kvh;
        if constexpr (KV4) {
          const uint8_t *kr = (const uint8_t *)a.k_pages + head * kv4::record_bytes(HD), *vr = (const uint8_t *)a.v_pages + head * kv4::record_bytes(HD);
          float dot = 0.f;
          for (int c = 0; c < HD; c += 8) {
            const int code = kv4::word_at(pos % 64, c / 8), pair = kv4::code_bytes(HD) + (pos % 64 * (HD / 32) + c / 32) * 4;
            const uint32_t kp = *reinterpret_cast<const uint32_t *>(kr + pair), vp = *reinterpret_cast<const uint32_t *>(vr + pair);
            uint32_t x[4], y[4];
            kv4::values8(*reinterpret_cast<const uint32_t *>(kr + code), kv4::low_twice(kp), kv4::high_twice(kp), x);
            kv4::values8(*reinterpret_cast<const uint32_t *>(vr + code), kv4::low_twice(vp), kv4::high_twice(vp), y);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 f = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162 *>(&x[e])), g = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162 *>(&y[e]));
              dot = fmaf(f.x, qs[c + 2 * e], dot); dot = fmaf(f.y, qs[c + 2 * e + 1], dot);
              vs[lane][c + 2 * e] = g.x; vs[lane][c + 2 * e + 1] = g.y;
            }
          }
          sc = dot; live = true;
        } else {
          row_of((const bf16 *)a.k_pages + (head * 64 + pos % 64) * HD, (const bf16 *)a.v_pages + (head * 64 + pos % 64) * HD);
        }
      }
    } else if (t < total) {
      const long long at = (w.loc0 + (t - n_sink - n_window)) * a.local_stride + kvh * HD;
      row_of(a.k_local + at, a.v_local + at);
    }
    const float top = fmaxf(mx, warp_max(sc));
    const float keep = top == -INFINITY ? 1.f : __expf(mx - top);
    const float p = live ? __expf(sc - top) : 0.f;
    den = den * keep + warp_sum(p);
#pragma unroll
    for (int i = 0; i < DPL; ++i) acc[i] *= keep;
    mx = top;
    const unsigned seen = __ballot_sync(0xffffffffu, live);
    for (int j = 0; j < 32; ++j) {
      const float pj = __shfl_sync(0xffffffffu, p, j);
      if (!(seen >> j & 1)) continue;
#pragma unroll
      for (int i = 0; i < DPL; ++i) acc[i] = fmaf(pj, vs[j][lane + 32 * i], acc[i]);
    }
    __syncwarp();
  }
  bf16 *o = a.out + ((size_t)r * a.Hq + h) * HD;
#pragma unroll
  for (int i = 0; i < DPL; ++i) o[lane + 32 * i] = __float2bfloat16(den > 0.f ? acc[i] / den : 0.f);      // no visible key: zeros
}
