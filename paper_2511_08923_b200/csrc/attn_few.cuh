// Attention of few rows per KV head over 4-bit pages: single tokens, short causal runs, the shortest blocks.
//
// Such calls are bound by reading the cache, 5/8 of a byte per element, so what a key costs beyond that has to stay small: one page of a head
// (64 keys, 10 KB for head_dim 128) passes an SM in about 230 ns at the memory's rate.  The 128-row tiles of the tcgen05 kernel would spend 500 ns
// of tensor work on it, most of it on empty rows, and a trip of every key through shared memory in bf16.  Here a warp keeps 8 or 16 rows (query heads of a KV
// head times slots) as the narrow operand of mma.sync (S^T = K Q^T, O^T = V^T P^T: keys and dimensions are the tall one) and turns codes into
// fragments in its own registers.  The order of the dimensions in K Q^T and of the keys in V^T P^T does not matter to a sum, so both are chosen
// such that a lane's operands are what it reads with one wide load, and no value ever goes back to shared memory.
//   K Q^T: lane (g, t) = (lane / 4, lane % 4) reads head_dim / 4 dimensions, from t head_dim / 4 on, of the keys that are rows g and g + 8; step i of
//     the product takes four of them (two register pairs).  With head_dim 128 they are one group: one scale, one base.
//   P goes from "key g, rows 2 t and 2 t + 1" to "keys 2 t and 2 t + 1, row g" by transposing 8 x 8 matrices of bf16 (movmatrix).
//   V^T P^T: the lane reads head_dim / 8 dimensions, from g head_dim / 8 on, of four keys (t, t + 4, t + 8, t + 12 of 16) and pairs them key by key; two of
//     those dimensions are rows g and g + 8 of an output tile.  Keys are numbered accordingly: row 2 t of a score tile is key t, row 2 t + 1 is key t + 4.
// Chunks of 32 keys arrive through cp.async into a ring of the warp's own, one chunk ahead; there is no barrier between warps until a unit's end.
//
// Work distribution: units (sequence, KV head, tile of rows) have as many chunks as their sequence's rows see; all chunks of the call, unit after
// unit, are cut into equal shares, one per CTA, whose four warps take chunks in turn.  Where a share ends inside a unit, partial results (maximum,
// sum, O) go to scratch, and the CTA that delivers a unit's last one merges them in the order of the shares (so that results do not depend on
// who that is).  Nothing waits for another CTA.
#pragma once
#include <type_traits>
#include "common.cuh"
#include "kernels_cache.cuh"
#include "sm100_ptx.cuh"

namespace attn_few {

constexpr int WARPS = 4, CHUNK = 32, MAX_ROWS = 16, MAX_CTAS_PER_SM = 3;
constexpr float RAISE_THRESHOLD = 8.f;                 // log2 units (as in attn_tc.cuh)
constexpr int AT_ONCE = 12;                            // partial results of a unit read at once
// CTAs per SM, for 8 n8 rows: what the registers allow.  With 8 rows there are two instances: three CTAs fill an SM's pipes better, two have the registers to
// overlap more of a chunk's work (24 sequences of up to 16 k positions 75 and 81 us, one of 32 k 27 and 23).
__host__ __device__ constexpr int ctas_per_sm(int n8, bool many) { return n8 == 1 && many ? 3 : 2; }

template <int HD, int N8>
struct Smem {
  // A chunk: the groups' codes (32 rows of 16 bytes each) as far apart as lets a warp's loads of K or of V reach all banks, then the pairs; K, then V.
  static constexpr int PLANES = HD / 32, K_PLANE = 512 + (HD == 128 ? 16 : 32), V_PLANE = 512 + 64, PAIRS = CHUNK * PLANES * 4;
  static constexpr int V_OFF = PLANES * K_PLANE + PAIRS, STAGE = V_OFF + PLANES * V_PLANE + PAIRS;
  static constexpr int RING = 2 * STAGE;                                                               // two chunks per warp
  static constexpr int O_REGS = HD / 4 * N8, STATS = 4 * N8;                                           // per lane: O; maxima and sums of two rows of each eight
  static constexpr int MERGE_OFF = WARPS * RING, MERGE_BYTES = (O_REGS + STATS) * 32 * 4;
  static constexpr int TOTAL = MERGE_OFF + 2 * MERGE_BYTES;
};
static_assert(Smem<128, 1>::TOTAL * ctas_per_sm(1, true) <= 224 * 1024 && Smem<128, 2>::TOTAL * ctas_per_sm(2, true) <= 224 * 1024, "CTAs of an SM fit its shared memory");

struct Args {
  CacheArgs c;
  int n_seqs, tiles, ctas, most;      // tiles of 8 n8 rows per (sequence, KV head); CTAs that take shares at most, and in calls of fewer than 16 chunks per warp
  float scale_log2;
  float *part_O; float2 *part_ml;     // [2 CTAs][MAX_ROWS][HD], [2 CTAs][MAX_ROWS]
  int32_t *arrived;                   // [CTAs], zero between calls: partial results of the split unit that begins in that CTA's share
};

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {      // of an 8 x 8 matrix of 16-bit elements, lane (g, t) holding row g, columns 2 t and 2 t + 1
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src, bool live) {      // !live: zeros, nothing is read
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(live ? BYTES : 0) : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t *>(&h);
}

// The chunks that the rows of a sequence of n cached positions see between them: [0, sink) and [first, end) of the cache, then local rows.
struct Chunks { int n, sink, skip, cached, all; };       // cached ones: c < sink ? c : c + skip; local ones behind them
__device__ __forceinline__ Chunks chunks_of(const WindowRows &w, int n) {
  Chunks c{n, 0, 0, 0, 0};
  if (n < 0) return c;
  c.cached = (int)(((long long)n + w.k + CHUNK - 1) / CHUNK);
  if (w.window > 0) {
    const int first = max(n - w.window + 1, 0) / CHUNK;                   // the first slot's window reaches furthest back
    c.sink = min((int)(((long long)w.sinks + CHUNK - 1) / CHUNK), first);
    c.skip = first - c.sink; c.cached -= c.skip;
  }
  c.all = c.cached + (w.blocks ? (w.k * w.k + CHUNK - 1) / CHUNK : 0);
  return c;
}

template <int HD, int N8, bool MANY>
__global__ void __launch_bounds__(WARPS * 32, ctas_per_sm(N8, MANY)) attn_few_kernel(const Args a) {
  using L = Smem<HD, N8>;
  constexpr int ROWS = 8 * N8, QK = HD / 16, DT = HD / 4, MT = HD / 16, DV = HD / 8;      // steps of K Q^T; dimensions a lane reads of a key of K; output tiles; dimensions it reads of a key of V
  extern __shared__ __align__(128) uint8_t few_smem[];
  __shared__ long long sums[WARPS][4], sum_s[WARPS];
  __shared__ long long found_base;
  __shared__ int found_seq, is_last;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const WindowRows &wr = a.c.rows;
  const int T = wr.rows(), G = a.c.Hq / a.c.Hkv, per_seq = a.c.Hkv * a.tiles;      // units per sequence
  pdl_trigger();
  pdl_wait();

  // ---- this CTA's share [w0, w1) of all chunks ----
  auto length = [&](int s) { return min(wr.seq_len[s], wr.n_max); };
  const int all0 = threadIdx.x < a.n_seqs ? chunks_of(wr, length(threadIdx.x)).all : 0;       // of this thread's sequence among the first ones
  auto all_of = [&](int s) { return s < WARPS * 32 ? all0 : chunks_of(wr, length(s)).all; };    // (s = this thread's)
  // Shares.  While the SMs are not full a warp takes about 1 us per chunk, and merging a unit's p parts 0.15 p us (for that many trips to the L2):
  // chunks / (4 p) + 0.15 p is least for p = sqrt(1.7 chunks) (12/2 heads, 8 k positions: 63 parts 22.3 us, 31: 17.6, 16: 17.2).  Where two CTAs per SM hold
  // such parts of all units, those are the shares: one that ends a unit and begins another takes twice as long (32 sequences of up to 200 positions: 14.1 us
  // with shares that do, 9.5 without).  Otherwise shares are even, across units.
  int parts_most = 0x7fffffff;
  auto parts = [&](int all) { return all == 0 ? 0 : min(min((all + WARPS - 1) / WARPS, parts_most), max(1, (int)sqrtf(1.7f * (float)all))); };
  long long chunks = 0, n_parts_all = 0, units = 0;
  int longest = 0;
  for (int s = threadIdx.x; s < a.n_seqs; s += WARPS * 32) {
    const int all = all_of(s);
    chunks += all; n_parts_all += parts(all); units += all > 0; longest = max(longest, all);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    chunks += __shfl_xor_sync(0xffffffffu, chunks, o); n_parts_all += __shfl_xor_sync(0xffffffffu, n_parts_all, o); units += __shfl_xor_sync(0xffffffffu, units, o);
    longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, o));
  }
  if (lane == 0) { sums[warp][0] = chunks; sums[warp][1] = n_parts_all; sums[warp][2] = units; sums[warp][3] = longest; }
  __syncthreads();
  const long long W = (sums[0][0] + sums[1][0] + sums[2][0] + sums[3][0]) * per_seq;
  n_parts_all = (sums[0][1] + sums[1][1] + sums[2][1] + sums[3][1]) * per_seq; units = (sums[0][2] + sums[1][2] + sums[2][2] + sums[3][2]) * per_seq;
  longest = (int)max(max(sums[0][3], sums[1][3]), max(sums[2][3], sums[3][3]));
  bool even = n_parts_all > a.most;
  int C = (int)min((W + WARPS - 1) / WARPS, (long long)(W >= 16ll * WARPS * a.ctas ? a.ctas : a.most));
  if (even && units <= a.most) {                       // fewer parts of each unit, where the longest one's then take no longer than even shares and 3 us
    const int p = a.most / (int)max(units, 1ll);
    if ((float)longest <= (float)W * (float)p / (float)a.most + 12.f * (float)p) { even = false; parts_most = p; n_parts_all = min(units * p, (long long)a.most); }
  }
  if (!even) C = (int)n_parts_all;                     // (with fewer parts than that the last ones find nothing)
  if ((int)blockIdx.x >= C) return;
  const long long w0 = even ? W * blockIdx.x / C : blockIdx.x;       // the share's first chunk among all; or its number
  if (threadIdx.x == 0) found_seq = -1;
  {                                                    // the sequence that it lies in
    long long base = 0;
    for (int s0 = 0; s0 < a.n_seqs; s0 += WARPS * 32) {
      const int s = s0 + threadIdx.x, all = s < a.n_seqs ? all_of(s) : 0;
      const long long work = (long long)(even ? all : parts(all)) * per_seq;
      long long incl = work;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const long long x = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += x; }
      __syncthreads();
      if (lane == 31) sum_s[warp] = incl;
      __syncthreads();
      for (int v = 0; v < warp; ++v) incl += sum_s[v];
      const long long lo = base + incl - work, hi = base + incl;
      if (lo <= w0 && w0 < hi) { found_seq = s; found_base = lo; }
      base += sum_s[0] + sum_s[1] + sum_s[2] + sum_s[3];
      if (base > w0) break;
    }
    __syncthreads();
    if (found_seq < 0) return;
  }

  // A place among the chunks: chunk c of unit `unit` of sequence `seq`.
  struct Place { int seq, unit, c; Chunks ch; };
  Place here;                                          // of the share's unit that is being worked on
  here.seq = found_seq; here.ch = chunks_of(wr, length(here.seq));
  int share, part0 = 0, n_parts = 1;                   // its chunks; a unit's parts are those of CTAs part0 .. part0 + n_parts - 1
  if (even) {
    here.unit = (int)((w0 - found_base) / here.ch.all); here.c = (int)(w0 - found_base - (long long)here.unit * here.ch.all);
    share = (int)(W * (blockIdx.x + 1) / C - w0);
  } else {
    n_parts = parts(here.ch.all);
    here.unit = (int)(w0 - found_base) / n_parts;
    part0 = (int)found_base + here.unit * n_parts;
    const int j = blockIdx.x - part0;
    here.c = (int)((long long)here.ch.all * j / n_parts);
    share = (int)((long long)here.ch.all * (j + 1) / n_parts) - here.c;
  }
  auto advance = [&](Place &p, int by) {               // (there is such a place)
    p.c += by;
    while (p.c >= p.ch.all) {
      p.c -= p.ch.all;
      if (++p.unit == per_seq) { p.unit = 0; do { ++p.seq; p.ch = chunks_of(wr, length(p.seq)); } while (p.ch.all == 0); }
    }
  };

  // ---- what a warp fetches: chunks warp, warp + 4, ... of the share ----
  struct Piece { int kind, at; };                      // kind 0: cached keys from position `at` on, 1: local rows from `at` on, -1: nothing to see
  constexpr int PB = L::PLANES * 4;
  const uint32_t ring = sm100::smem_u32(few_smem) + warp * L::RING + lane * 16, ring_pairs = sm100::smem_u32(few_smem) + warp * L::RING + lane * PB;
  const uint8_t *const k_codes = (const uint8_t *)a.c.k_pages + lane * 16, *const v_codes = (const uint8_t *)a.c.v_pages + lane * 16;
  const uint8_t *const k_pairs = (const uint8_t *)a.c.k_pages + kv4::code_bytes(HD) + lane * PB, *const v_pairs = (const uint8_t *)a.c.v_pages + kv4::code_bytes(HD) + lane * PB;
  Place f = here;                                      // of the chunk that is fetched next, number f_at of the share
  int f_at = warp, f_page = -1;                        // its page, read when the chunk before it was fetched
  auto chunk_of = [&](const Place &p) { return p.c < p.ch.sink ? p.c : p.c + p.ch.skip; };
  auto look_up = [&] { f_page = f_at < share && f.c < f.ch.cached ? a.c.table[(size_t)f.seq * a.c.width + (chunk_of(f) >> 1)] : -1; };
  if (f_at < share) advance(f, warp);
  look_up();
  auto fetch = [&](int stage) {
    Piece p{-1, 0};
    if (f_at >= share) return p;
    if (f.c >= f.ch.cached) { p.kind = 1; p.at = (f.c - f.ch.cached) * CHUNK; }
    else {
      const int chunk = chunk_of(f);
      p.at = chunk * CHUNK;
      if ((unsigned)f_page < (unsigned)a.c.n_pages) {
        p.kind = 0;
        const int kvh = a.tiles == 1 ? f.unit : f.unit / a.tiles, half = chunk & 1;
        const size_t rec = ((size_t)f_page * a.c.Hkv + kvh) * kv4::record_bytes(HD) + half * 512, pairs = rec + half * (L::PAIRS - 512);
        const uint32_t dst = ring + stage * L::STAGE, dst_pairs = ring_pairs + stage * L::STAGE;
#pragma unroll
        for (int i = 0; i < L::PLANES; ++i) {
          copy_async<16>(dst + i * L::K_PLANE, k_codes + rec + i * 1024, true);
          copy_async<16>(dst + L::V_OFF + i * L::V_PLANE, v_codes + rec + i * 1024, true);
        }
        // a key that no row sees may hold anything: with a scale and a base of zero it stands for zeros
        bool seen = true;
        if (p.at + CHUNK > f.ch.n + wr.k || (wr.window > 0 && p.at <= f.ch.n - wr.window)) {
          const int pos = p.at + lane;
          seen = pos < f.ch.n + wr.k && (wr.window == 0 || pos < wr.sinks || pos > f.ch.n - wr.window);
        }
        copy_async<PB>(dst_pairs + L::PLANES * L::K_PLANE, k_pairs + pairs, seen);
        copy_async<PB>(dst_pairs + L::V_OFF + L::PLANES * L::V_PLANE, v_pairs + pairs, seen);
      }
    }
    f_at += WARPS;
    if (f_at < share) advance(f, WARPS);
    look_up();
    return p;
  };
  auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };
  int next_at = warp;                                  // number, in the share, of the piece that was fetched last
  int stage = 0;
  Piece next = fetch(0);
  commit();

  // ---- units of the share, one after the other ----
  for (int done = 0; done < share;) {
    const int all = here.ch.all, len = min(all - here.c, share - done), kvh = here.unit / a.tiles, tile = here.unit - kvh * a.tiles, seq = here.seq, n = here.ch.n;
    const bool begins = here.c == 0, cut = !begins || here.c + len < all;
    const int rows_here = min(T * G - tile * ROWS, ROWS), row0 = tile * ROWS;
    const int n_local = wr.k * wr.k;
    // query rows g of every eight as fragments
    uint32_t q[N8][QK][2];
#pragma unroll
    for (int r = 0; r < N8; ++r) {
      const int m = row0 + 8 * r + g, slot = m / G;
      const bf16 *src = a.c.q + ((long long)seq * T + slot) * a.c.q_stride + (kvh * G + (m - slot * G)) * HD + t * DT;
#pragma unroll
      for (int i = 0; i < QK / 2; ++i) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (8 * r + g < rows_here) u = *reinterpret_cast<const uint4 *>(src + i * 8);
        q[r][2 * i][0] = u.x; q[r][2 * i][1] = u.y; q[r][2 * i + 1][0] = u.z; q[r][2 * i + 1][1] = u.w;
      }
    }
    // what rows 2 t and 2 t + 1 of every eight see; a row that is not there sees everything, so that nothing is masked for it
    int nvis[N8][2], low[N8][2], loc[N8][2];
#pragma unroll
    for (int r = 0; r < N8; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int m = row0 + 8 * r + 2 * t + h, slot = m / G;
        nvis[r][h] = 0x7fffffff; low[r][h] = 0; loc[r][h] = 0x7fffffff;
        if (8 * r + 2 * t + h < rows_here) {
          nvis[r][h] = n + slot + 1; loc[r][h] = -1;
          int pos = n + slot;
          if (slot >= wr.k) {
            const int b = (slot - wr.k) / wr.k;
            nvis[r][h] = n + b + 1; pos = n + b + 1 + (slot - wr.k - b * wr.k); loc[r][h] = b * wr.k;
          }
          low[r][h] = wr.window > 0 ? max(pos - wr.window + 1, 0) : 0;
        }
      }
    float o[N8][MT][4], m_ref[N8][2], l_run[N8][2];
#pragma unroll
    for (int r = 0; r < N8; ++r) {
      m_ref[r][0] = m_ref[r][1] = -INFINITY; l_run[r][0] = l_run[r][1] = 0.f;
#pragma unroll
      for (int i = 0; i < MT; ++i) o[r][i][0] = o[r][i][1] = o[r][i][2] = o[r][i][3] = 0.f;
    }

    // one chunk: cached keys whose codes are at kb and vb, the first one at position at0; or local rows from at0 on
    auto work = [&](auto is_local, int at0, const uint8_t *kb, const uint8_t *vb) {
      constexpr bool LOCAL = decltype(is_local)::value;
      // scores: tile j has keys 16 j ..; row g of its first and second half is key (g / 2) + 4 (g & 1)
      float s[N8][2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint32_t b[2][DT / 2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int key = 16 * j + 8 * h + (g >> 1) + 4 * (g & 1);
          if constexpr (!LOCAL) {
            const uint32_t sb = *reinterpret_cast<const uint32_t *>(kb + L::PLANES * L::K_PLANE + (key * L::PLANES + t * DT / 32) * 4);
            const uint32_t ss = kv4::low_twice(sb), bb = kv4::high_twice(sb);
            uint32_t w[DT / 8];
            if constexpr (HD == 128) { const uint4 u = *reinterpret_cast<const uint4 *>(kb + t * L::K_PLANE + key * 16); w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w; }
            else { const uint2 u = *reinterpret_cast<const uint2 *>(kb + (t >> 1) * L::K_PLANE + key * 16 + (t & 1) * 8); w[0] = u.x; w[1] = u.y; }
#pragma unroll
            for (int i = 0; i < DT / 8; ++i) {
              uint32_t x[4];
              kv4::values8(w[i], ss, bb, x);
              b[h][4 * i] = x[0]; b[h][4 * i + 1] = x[1]; b[h][4 * i + 2] = x[2]; b[h][4 * i + 3] = x[3];
            }
          } else {
            const bool live = at0 + key < n_local;
            const bf16 *src = a.c.k_local + ((long long)seq * n_local + at0 + key) * a.c.local_stride + kvh * HD + t * DT;
#pragma unroll
            for (int i = 0; i < DT / 8; ++i) {
              uint4 u = make_uint4(0, 0, 0, 0);
              if (live) u = *reinterpret_cast<const uint4 *>(src + i * 8);
              b[h][4 * i] = u.x; b[h][4 * i + 1] = u.y; b[h][4 * i + 2] = u.z; b[h][4 * i + 3] = u.w;
            }
          }
        }
#pragma unroll
        for (int r = 0; r < N8; ++r) {
          s[r][j][0] = s[r][j][1] = s[r][j][2] = s[r][j][3] = 0.f;
#pragma unroll
          for (int i = 0; i < QK; ++i) {
            const uint32_t x[4] = {b[0][2 * i], b[1][2 * i], b[0][2 * i + 1], b[1][2 * i + 1]};
            mma(s[r][j], x, q[r][i][0], q[r][i][1]);
          }
        }
      }
      // whether every row sees all of the chunk: slot 0 sees the fewest positions, and no slot is further ahead than n + 2 k - 1
      const bool whole = !LOCAL && at0 + CHUNK <= n + 1 && (wr.window == 0 || at0 > n + 2 * wr.k - 1 - wr.window || at0 + CHUNK <= wr.sinks);
      uint32_t p[N8][2][2];
#pragma unroll
      for (int r = 0; r < N8; ++r) {
        if (!whole) {
          // a row sees keys [0, skip) and [lo, hi) of the chunk; element e of tile j: row 2 t + (e & 1), key 16 j + 8 (e / 2) + (g / 2) + 4 (g & 1)
          int lo[2], hi[2], skip[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if constexpr (!LOCAL) { hi[h] = nvis[r][h] - at0; lo[h] = low[r][h] - at0; skip[h] = min(wr.sinks - at0, hi[h]); }
            else {
              const int first = loc[r][h];             // (-1: sees no local rows)
              lo[h] = first < 0 ? CHUNK : first - at0; hi[h] = first < 0 ? 0 : lo[h] + wr.k; skip[h] = 0;
              if (first == 0x7fffffff) { lo[h] = 0; hi[h] = CHUNK; }
            }
          }
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int h = e & 1, key = 16 * j + 8 * (e >> 1) + (g >> 1) + 4 * (g & 1);
              if (!(key < skip[h] || (key >= lo[h] && key < hi[h]))) s[r][j][e] = -INFINITY;
            }
        }
        // softmax in base 2; the reference rises only when it is exceeded by the threshold
        float m_new[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float mx = fmaxf(sm100::max3(s[r][0][h], s[r][0][2 + h], s[r][1][h]), s[r][1][2 + h]);
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16)) * a.scale_log2;
          m_new[h] = mx > m_ref[r][h] + RAISE_THRESHOLD ? mx : m_ref[r][h];
        }
        if (__any_sync(0xffffffffu, m_new[0] != m_ref[r][0] || m_new[1] != m_ref[r][1])) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float keep = m_new[h] == m_ref[r][h] ? 1.f : exp2f(m_ref[r][h] - m_new[h]);
            l_run[r][h] *= keep;
#pragma unroll
            for (int i = 0; i < MT; ++i) { o[r][i][h] *= keep; o[r][i][2 + h] *= keep; }
            m_ref[r][h] = m_new[h];
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float neg = m_ref[r][h] == -INFINITY ? 0.f : -m_ref[r][h];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            s[r][j][h] = sm100::ex2_approx(fmaf(s[r][j][h], a.scale_log2, neg)); s[r][j][2 + h] = sm100::ex2_approx(fmaf(s[r][j][2 + h], a.scale_log2, neg));
            l_run[r][h] += s[r][j][h] + s[r][j][2 + h];
          }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {                    // (the matrix instruction takes the weights in bf16; their sum is kept of the 32-bit ones: a weight is off by 2^-8 of itself at most)
          p[r][j][0] = transposed(pack_bf16(s[r][j][0], s[r][j][1]));
          p[r][j][1] = transposed(pack_bf16(s[r][j][2], s[r][j][3]));
        }
      }
      // V^T P^T, eight of a lane's dimensions (four output tiles) at a time
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int k0 = 16 * j + t;                      // the lane's keys: k0, k0 + 4 | k0 + 8, k0 + 12
        uint32_t w[4][DV / 8], ss[2], bb[2];
        if constexpr (!LOCAL) {
          const uint8_t *codes = vb + g * DV / 32 * L::V_PLANE + g * DV % 32 / 2, *pairs = vb + L::PLANES * L::V_PLANE + g * DV / 32 * 4;
          uint32_t sb[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (HD == 128) { const uint2 u = *reinterpret_cast<const uint2 *>(codes + (k0 + 4 * e) * 16); w[e][0] = u.x; w[e][1] = u.y; }
            else w[e][0] = *reinterpret_cast<const uint32_t *>(codes + (k0 + 4 * e) * 16);
            sb[e] = *reinterpret_cast<const uint32_t *>(pairs + (k0 + 4 * e) * (L::PLANES * 4));
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) { ss[h] = __byte_perm(sb[2 * h], sb[2 * h + 1], 0x5410); bb[h] = __byte_perm(sb[2 * h], sb[2 * h + 1], 0x7632); }
        }
#pragma unroll
        for (int d = 0; d < DV / 8; ++d) {
          uint32_t b[2][8];                             // [pair of keys][dimension]
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t x[4], y[4];                        // the even dimensions of both keys side by side, the odd ones
            if constexpr (!LOCAL) {
              kv4::values8(__byte_perm(w[2 * h][d], w[2 * h + 1][d], 0x5410), ss[h], bb[h], x);
              kv4::values8(__byte_perm(w[2 * h][d], w[2 * h + 1][d], 0x7632), ss[h], bb[h], y);
            } else {
              const int ka = at0 + k0 + 8 * h, kc = ka + 4;
              const bf16 *src = a.c.v_local + (long long)seq * n_local * a.c.local_stride + kvh * HD + g * DV + d * 8;
              uint4 u = make_uint4(0, 0, 0, 0), v = u;
              if (ka < n_local) u = *reinterpret_cast<const uint4 *>(src + ka * a.c.local_stride);
              if (kc < n_local) v = *reinterpret_cast<const uint4 *>(src + kc * a.c.local_stride);
              x[0] = __byte_perm(u.x, v.x, 0x5410); x[1] = __byte_perm(u.y, v.y, 0x5410); x[2] = __byte_perm(u.z, v.z, 0x5410); x[3] = __byte_perm(u.w, v.w, 0x5410);
              y[0] = __byte_perm(u.x, v.x, 0x7632); y[1] = __byte_perm(u.y, v.y, 0x7632); y[2] = __byte_perm(u.z, v.z, 0x7632); y[3] = __byte_perm(u.w, v.w, 0x7632);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) { b[h][2 * e] = x[e]; b[h][2 * e + 1] = y[e]; }
          }
#pragma unroll
          for (int r = 0; r < N8; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t x[4] = {b[0][2 * e], b[0][2 * e + 1], b[1][2 * e], b[1][2 * e + 1]};
              mma(o[r][4 * d + e], x, p[r][j][0], p[r][j][1]);
            }
        }
      }
    };
    while (next_at < done + len) {
      const Piece cur = next;
      next_at += WARPS;
      __syncwarp();                                    // (all lanes are done with the stage that is filled now)
      next = fetch(stage ^ 1);
      commit();
      asm volatile("cp.async.wait_group 1;" ::: "memory");
      __syncwarp();
      const uint8_t *kb = few_smem + warp * L::RING + stage * L::STAGE;
      stage ^= 1;
      if (cur.kind == 0) work(std::false_type{}, cur.at, kb, kb + L::V_OFF);
      else if (cur.kind == 1) work(std::true_type{}, cur.at, kb, kb);
    }

    // ---- the four warps' results: 2 and 3 to 0 and 1, then 1 to 0 ----
#pragma unroll
    for (int r = 0; r < N8; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l_run[r][h] += __shfl_xor_sync(0xffffffffu, l_run[r][h], x);
    auto hand_over = [&](int area) {
      float *x = reinterpret_cast<float *>(few_smem + L::MERGE_OFF + area * L::MERGE_BYTES) + lane;
#pragma unroll
      for (int r = 0; r < N8; ++r) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[((r * MT + i) * 4 + e) * 32] = o[r][i][e];
#pragma unroll
        for (int h = 0; h < 2; ++h) { x[(L::O_REGS + 4 * r + h) * 32] = m_ref[r][h]; x[(L::O_REGS + 4 * r + 2 + h) * 32] = l_run[r][h]; }
      }
    };
    auto take_over = [&](int area) {
      const float *x = reinterpret_cast<const float *>(few_smem + L::MERGE_OFF + area * L::MERGE_BYTES) + lane;
#pragma unroll
      for (int r = 0; r < N8; ++r) {
        float mine_w[2], other_w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float other = x[(L::O_REGS + 4 * r + h) * 32], M = fmaxf(m_ref[r][h], other);
          mine_w[h] = m_ref[r][h] == -INFINITY ? 0.f : exp2f(m_ref[r][h] - M); other_w[h] = other == -INFINITY ? 0.f : exp2f(other - M);
          l_run[r][h] = mine_w[h] * l_run[r][h] + other_w[h] * x[(L::O_REGS + 4 * r + 2 + h) * 32];
          m_ref[r][h] = M;
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[r][i][e] = mine_w[e & 1] * o[r][i][e] + other_w[e & 1] * x[((r * MT + i) * 4 + e) * 32];
      }
    };
    if (warp >= 2) hand_over(warp - 2);
    __syncthreads();
    if (warp < 2) take_over(warp);
    if (warp == 1) hand_over(1);
    __syncthreads();
    int first_cta = part0, last_cta = part0 + n_parts - 1;         // those whose shares the unit's first and last chunk lie in
    if (even && cut) {
      const long long u0 = w0 + done - here.c, u1 = u0 + all;
      first_cta = (int)(((u0 + 1) * C - 1) / W); last_cta = (int)((u1 * C - 1) / W);
    }
    if (warp == 0) {
      take_over(1);
#pragma unroll
      for (int r = 0; r < N8; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = 8 * r + 2 * t + h, m = row0 + row, slot = m / G;
          if (row >= rows_here) continue;
          // dimensions g DV .. + DV: tile i has two of them
          if (!cut) {
            const float inv = l_run[r][h] > 0.f ? 1.f / l_run[r][h] : 0.f;         // (a row that sees nothing: zeros)
            bf16 *dst = a.c.out + (((long long)seq * T + slot) * a.c.Hq + kvh * G + (m - slot * G)) * HD + g * DV;
#pragma unroll
            for (int i = 0; i < MT; i += 4) {
              uint4 u;
              u.x = pack_bf16(o[r][i][h] * inv, o[r][i][2 + h] * inv); u.y = pack_bf16(o[r][i + 1][h] * inv, o[r][i + 1][2 + h] * inv);
              u.z = pack_bf16(o[r][i + 2][h] * inv, o[r][i + 2][2 + h] * inv); u.w = pack_bf16(o[r][i + 3][h] * inv, o[r][i + 3][2 + h] * inv);
              *reinterpret_cast<uint4 *>(dst + 2 * i) = u;
            }
          } else {
            const size_t part = (size_t)(2 * blockIdx.x + begins) * MAX_ROWS + row;
            float *dst = a.part_O + part * HD + g * DV;
#pragma unroll
            for (int i = 0; i < MT; i += 2) *reinterpret_cast<float4 *>(dst + 2 * i) = make_float4(o[r][i][h], o[r][i][2 + h], o[r][i + 1][h], o[r][i + 1][2 + h]);
            if (g == 0) a.part_ml[part] = make_float2(m_ref[r][h], l_run[r][h]);
          }
        }
      if (cut) {
        __threadfence();
        __syncwarp();
        if (lane == 0) is_last = atomicAdd(&a.arrived[first_cta], 1) == last_cta - first_cta;
      }
    }
    __syncthreads();
    if (cut && is_last) {
      __threadfence();
      const int pieces = last_cta - first_cta + 1;
      for (int i = threadIdx.x; i < rows_here * (HD / 4); i += WARPS * 32) {
        const int r = i / (HD / 4), d = i % (HD / 4) * 4;
        auto part = [&](int x) { return (size_t)(2 * (first_cta + x) + (x == 0)) * MAX_ROWS + r; };
        float M = -INFINITY, den = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int x0 = 0; x0 < pieces; x0 += AT_ONCE) {      // their loads ahead of the first use: a trip to the L2 costs as much as all else
          float2 ml[AT_ONCE]; float4 v[AT_ONCE];
#pragma unroll
          for (int e = 0; e < AT_ONCE; ++e) {
            ml[e] = make_float2(-INFINITY, 0.f); v[e] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (x0 + e < pieces) { ml[e] = __ldcg(a.part_ml + part(x0 + e)); v[e] = __ldcg(reinterpret_cast<const float4 *>(a.part_O + part(x0 + e) * HD + d)); }
          }
          float top = M;
#pragma unroll
          for (int e = 0; e < AT_ONCE; ++e) top = fmaxf(top, ml[e].x);
          const float keep = M == -INFINITY ? 0.f : exp2f(M - top);
          M = top; den *= keep;
          acc.x *= keep; acc.y *= keep; acc.z *= keep; acc.w *= keep;
#pragma unroll
          for (int e = 0; e < AT_ONCE; ++e) {
            const float w = ml[e].x == -INFINITY ? 0.f : exp2f(ml[e].x - M);
            den += w * ml[e].y;
            acc.x = fmaf(w, v[e].x, acc.x); acc.y = fmaf(w, v[e].y, acc.y); acc.z = fmaf(w, v[e].z, acc.z); acc.w = fmaf(w, v[e].w, acc.w);
          }
        }
        const float inv = den > 0.f ? 1.f / den : 0.f;
        const int m = row0 + r, slot = m / G;
        uint2 u;
        u.x = pack_bf16(acc.x * inv, acc.y * inv); u.y = pack_bf16(acc.z * inv, acc.w * inv);
        *reinterpret_cast<uint2 *>(a.c.out + (((long long)seq * T + slot) * a.c.Hq + kvh * G + (m - slot * G)) * HD + d) = u;
      }
      if (threadIdx.x == 0) a.arrived[first_cta] = 0;
    }
    done += len;
    if (done < share) advance(here, len);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

}  // namespace attn_few
