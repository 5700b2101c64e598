// Attention of few rows per KV head over 4-bit pages: single tokens, short causal runs, the shortest blocks.
//
// Such calls are bound by reading the cache, 5/8 of a byte per element, so what a key costs beyond that has to stay small: one page of a head
// (64 keys, 10 KB for head_dim 128) passes an SM in about 230 ns at the memory's rate.  The 128-row tiles of the tcgen05 kernel would spend 500 ns
// of tensor work on it, most of it on empty rows, and a trip of every key through shared memory in bf16.  Here a warp keeps 16 rows (query heads of a KV head
// times slots) as mma.sync fragments and turns codes into operand fragments in its own registers: the order of the dimensions in Q K^T and of
// the keys in P V does not matter to a sum, so both are chosen such that a lane's operands are what it reads with one wide load, and no value
// ever goes back to shared memory.
//   Q K^T: lane (g, t) = (lane / 4, lane % 4) reads head_dim / 4 dimensions, from t head_dim / 4 on, of the key that is column g; step i of the
//     product takes four of them (two register pairs).  With head_dim 128 they are one group: one scale, one base.
//   P V: the lane reads head_dim / 8 dimensions, from g head_dim / 8 on, of four keys (t, t + 4, t + 8, t + 12 of 16), pairs them key by key, and each of
//     those dimensions is column g of an output tile of its own.  The keys of a score tile are numbered accordingly: column 2 t is key t, 2 t + 1 is t + 4.
// Chunks of 32 keys arrive through cp.async into a ring of the warp's own, one chunk ahead; there is no barrier between warps until a unit's end.
//
// Work distribution: units (sequence, KV head, tile of 16 rows) have as many chunks as their sequence's rows see; all chunks of the call, unit after
// unit, are cut into equal shares, one per CTA, whose four warps take chunks in turn.  Where a share ends inside a unit, partial results (maximum,
// sum, O) go to scratch, and the CTA that delivers a unit's last one merges them in the order of the shares (so that results do not depend on
// who that is).  Nothing waits for another CTA.
#pragma once
#include "common.cuh"
#include "kernels_cache.cuh"
#include "sm100_ptx.cuh"

namespace attn_few {

constexpr int WARPS = 4, CHUNK = 32, ROWS = 16, CTAS_PER_SM = 3;
constexpr float RAISE_THRESHOLD = 8.f;                 // log2 units (as in attn_tc.cuh)

template <int HD>
struct Smem {
  // A chunk: the groups' codes (32 rows of 16 bytes each) as far apart as lets a warp's loads of K or of V reach all banks, then the pairs; K, then V.
  static constexpr int PLANES = HD / 32, K_PLANE = 512 + (HD == 128 ? 16 : 32), V_PLANE = 512 + 64, PAIRS = CHUNK * PLANES * 4;
  static constexpr int V_OFF = PLANES * K_PLANE + PAIRS, STAGE = V_OFF + PLANES * V_PLANE + PAIRS;
  static constexpr int RING = 2 * STAGE;                                                               // two chunks per warp
  static constexpr int O_REGS = HD / 2;                                                                 // per lane
  static constexpr int MERGE_OFF = WARPS * RING, MERGE_BYTES = (O_REGS + 4) * 32 * 4;                   // one warp's O, maximum and sum
  static constexpr int TOTAL = MERGE_OFF + 3 * MERGE_BYTES;
};
static_assert(Smem<128>::TOTAL * CTAS_PER_SM <= 224 * 1024, "CTAs of an SM fit its shared memory");

struct Args {
  CacheArgs c;
  int n_seqs, tiles, ctas;            // tiles of 16 rows per (sequence, KV head); CTAs that take shares at most
  int per_warp;                       // chunks a warp has at least where there are enough
  float scale_log2;
  float *part_O; float2 *part_ml;     // [2 CTAs][16 rows][HD], [2 CTAs][16 rows]
  int32_t *arrived;                   // [CTAs], zero between calls: partial results of the split unit that begins in that CTA's share
};

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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
struct Chunks {
  int n, sink, first, end, local;
  __device__ __forceinline__ int cached() const { return sink + end - first; }
  __device__ __forceinline__ int all() const { return cached() + local; }
};
__device__ __forceinline__ Chunks chunks_of(const WindowRows &w, int n) {
  Chunks c{n, 0, 0, 0, 0};
  if (n < 0) return c;
  c.end = (int)(((long long)n + w.k + CHUNK - 1) / CHUNK);
  if (w.window > 0) {
    c.first = max(n - w.window + 1, 0) / CHUNK;                           // the first slot's window reaches furthest back
    c.sink = min((int)(((long long)w.sinks + CHUNK - 1) / CHUNK), c.first);
  }
  c.local = w.blocks ? (w.k * w.k + CHUNK - 1) / CHUNK : 0;
  return c;
}

template <int HD>
__global__ void __launch_bounds__(WARPS * 32, CTAS_PER_SM) attn_few_kernel(const Args a) {
  using L = Smem<HD>;
  constexpr int QK = HD / 16, DT = HD / 4, NT = HD / 8;      // steps of Q K^T; dimensions a lane reads of a key of K; output tiles (= dimensions it reads of a key of V)
  extern __shared__ __align__(128) uint8_t few_smem[];
  __shared__ long long sum_s[WARPS];
  __shared__ long long found_base;
  __shared__ int found_seq, is_last;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const WindowRows &wr = a.c.rows;
  const int T = wr.rows(), G = a.c.Hq / a.c.Hkv, per_seq = a.c.Hkv * a.tiles;      // units per sequence
  pdl_trigger();
  pdl_wait();

  // ---- this CTA's share [w0, w1) of all chunks ----
  auto length = [&](int s) { return min(wr.seq_len[s], wr.n_max); };
  auto block_sum = [&](long long v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if (lane == 0) sum_s[warp] = v;
    __syncthreads();
    return sum_s[0] + sum_s[1] + sum_s[2] + sum_s[3];
  };
  long long mine = 0;
  const int own0 = threadIdx.x < a.n_seqs ? chunks_of(wr, length(threadIdx.x)).all() * per_seq : 0;
  mine = own0;
  for (int s = threadIdx.x + WARPS * 32; s < a.n_seqs; s += WARPS * 32) mine += (long long)chunks_of(wr, length(s)).all() * per_seq;
  const long long W = block_sum(mine);
  const int C = (int)min((W + WARPS * a.per_warp - 1) / (WARPS * a.per_warp), (long long)a.ctas);
  if ((int)blockIdx.x >= C) return;
  const long long w0 = W * blockIdx.x / C, w1 = W * (blockIdx.x + 1) / C;
  {                                                    // the sequence that w0 lies in
    long long base = 0;
    for (int s0 = 0; s0 < a.n_seqs; s0 += WARPS * 32) {
      const int s = s0 + threadIdx.x;
      const long long work = s0 == 0 ? own0 : s < a.n_seqs ? (long long)chunks_of(wr, length(s)).all() * per_seq : 0;
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
  }

  // ---- what a warp fetches: chunks w0 + warp, w0 + warp + 4, ... ----
  struct Piece { int kind, at, cut; };                  // kind 0: cached keys from position `at` on, 1: local rows from `at` on, -1: nothing to see
  const uint32_t ring = sm100::smem_u32(few_smem) + warp * L::RING;
  int f_seq = found_seq;
  long long f_base = found_base, f_w = w0 + warp;
  Chunks f_ch = chunks_of(wr, length(f_seq));
  auto fetch = [&](int stage) {
    Piece p{-1, 0, 0};
    if (f_w >= w1) return p;
    while (f_w >= f_base + (long long)f_ch.all() * per_seq) { f_base += (long long)f_ch.all() * per_seq; ++f_seq; f_ch = chunks_of(wr, length(f_seq)); }
    const int in_seq = (int)(f_w - f_base), unit = in_seq / f_ch.all(), c = in_seq - unit * f_ch.all(), kvh = unit / a.tiles;
    f_w += WARPS;
    if (c >= f_ch.cached()) { p.kind = 1; p.at = (c - f_ch.cached()) * CHUNK; return p; }
    const int chunk = c < f_ch.sink ? c : f_ch.first + (c - f_ch.sink);
    p.at = chunk * CHUNK;
    const int page = a.c.table[(size_t)f_seq * a.c.width + (chunk >> 1)];
    if ((unsigned)page >= (unsigned)a.c.n_pages) return p;
    p.kind = 0;
    const size_t rec = ((size_t)page * a.c.Hkv + kvh) * kv4::record_bytes(HD);
    const uint8_t *k = (const uint8_t *)a.c.k_pages + rec, *v = (const uint8_t *)a.c.v_pages + rec;
    const int half = chunk & 1;
    // a key that no row sees may hold anything: with a scale and a base of zero it stands for zeros
    const int pos = p.at + lane;
    const bool seen = pos < f_ch.n + wr.k && (wr.window == 0 || pos < wr.sinks || pos > f_ch.n - wr.window);
    const uint32_t dst = ring + stage * L::STAGE;
#pragma unroll
    for (int i = 0; i < L::PLANES; ++i) {
      copy_async<16>(dst + i * L::K_PLANE + lane * 16, k + i * 1024 + half * 512 + lane * 16, true);
      copy_async<16>(dst + L::V_OFF + i * L::V_PLANE + lane * 16, v + i * 1024 + half * 512 + lane * 16, true);
    }
    constexpr int PB = L::PLANES * 4;
    copy_async<PB>(dst + L::PLANES * L::K_PLANE + lane * PB, k + kv4::code_bytes(HD) + half * L::PAIRS + lane * PB, seen);
    copy_async<PB>(dst + L::V_OFF + L::PLANES * L::V_PLANE + lane * PB, v + kv4::code_bytes(HD) + half * L::PAIRS + lane * PB, seen);
    return p;
  };
  auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };
  long long next_w = f_w;                               // of the piece that was fetched last
  int stage = 0;
  Piece next = fetch(0);
  commit();

  // ---- units of the share, one after the other ----
  int seq = found_seq;
  long long base = found_base;
  Chunks ch = chunks_of(wr, length(seq));
  for (long long a0 = w0; a0 < w1;) {
    while (a0 >= base + (long long)ch.all() * per_seq) { base += (long long)ch.all() * per_seq; ++seq; ch = chunks_of(wr, length(seq)); }
    const int unit = (int)(a0 - base) / ch.all(), kvh = unit / a.tiles, tile = unit - kvh * a.tiles;
    const long long u0 = base + (long long)unit * ch.all(), u1 = u0 + ch.all(), a1 = min(u1, w1);
    const int rows_here = min(T * G - tile * ROWS, ROWS);
    // this lane's rows g and g + 8: query fragments and what they see
    uint32_t q[QK][4];
    int nvis[2], low[2], loc[2], nloc[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = g + 8 * h, m = tile * ROWS + r, slot = m / G;
      nvis[h] = 0x7fffffff; low[h] = 0; loc[h] = 0; nloc[h] = 0x7fffffff;     // (a row that is not there sees everything, so that nothing is masked for it)
      if (r < rows_here) {
        nvis[h] = ch.n + slot + 1; nloc[h] = 0;
        int pos = ch.n + slot;
        if (slot >= wr.k) {
          const int b = (slot - wr.k) / wr.k;
          nvis[h] = ch.n + b + 1; pos = ch.n + b + 1 + (slot - wr.k - b * wr.k); loc[h] = b * wr.k; nloc[h] = wr.k;
        }
        low[h] = wr.window > 0 ? max(pos - wr.window + 1, 0) : 0;
      }
      const bf16 *src = a.c.q + ((long long)seq * T + slot) * a.c.q_stride + (kvh * G + (m - slot * G)) * HD + t * DT;
#pragma unroll
      for (int i = 0; i < QK / 2; ++i) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (r < rows_here) u = *reinterpret_cast<const uint4 *>(src + i * 8);
        q[2 * i][h] = u.x; q[2 * i][2 + h] = u.y; q[2 * i + 1][h] = u.z; q[2 * i + 1][2 + h] = u.w;
      }
    }
    float o[NT][4], m_ref[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

    while (next_w < a1) {
      const Piece cur = next;
      next_w += WARPS;
      __syncwarp();                                    // (all lanes are done with the stage that is filled now)
      next = fetch(stage ^ 1);
      commit();
      asm volatile("cp.async.wait_group 1;" ::: "memory");
      __syncwarp();
      const uint8_t *kb = few_smem + warp * L::RING + stage * L::STAGE, *vb = kb + L::V_OFF;
      stage ^= 1;
      if (cur.kind < 0) continue;
      // scores
      float s[4][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = 16 * (j >> 1) + (g >> 1) + 4 * (g & 1) + 8 * (j & 1);
        uint32_t b[DT / 2];
        if (cur.kind == 0) {
          const uint32_t sb = *reinterpret_cast<const uint32_t *>(kb + L::PLANES * L::K_PLANE + (key * L::PLANES + t * DT / 32) * 4);
          const uint32_t ss = kv4::low_twice(sb), bb = kv4::high_twice(sb);
          uint32_t w[DT / 8];
          if constexpr (HD == 128) { const uint4 u = *reinterpret_cast<const uint4 *>(kb + t * L::K_PLANE + key * 16); w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w; }
          else { const uint2 u = *reinterpret_cast<const uint2 *>(kb + (t >> 1) * L::K_PLANE + key * 16 + (t & 1) * 8); w[0] = u.x; w[1] = u.y; }
#pragma unroll
          for (int i = 0; i < DT / 8; ++i) {
            uint32_t x[4];
            kv4::values8(w[i], ss, bb, x);
            b[4 * i] = x[0]; b[4 * i + 1] = x[1]; b[4 * i + 2] = x[2]; b[4 * i + 3] = x[3];
          }
        } else {
          const bool live = cur.at + key < wr.k * wr.k;
          const bf16 *src = a.c.k_local + ((long long)seq * wr.k * wr.k + cur.at + key) * a.c.local_stride + kvh * HD + t * DT;
#pragma unroll
          for (int i = 0; i < DT / 8; ++i) {
            uint4 u = make_uint4(0, 0, 0, 0);
            if (live) u = *reinterpret_cast<const uint4 *>(src + i * 8);
            b[4 * i] = u.x; b[4 * i + 1] = u.y; b[4 * i + 2] = u.z; b[4 * i + 3] = u.w;
          }
        }
        s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
#pragma unroll
        for (int i = 0; i < QK; ++i) mma(s[j], q[i], b[2 * i], b[2 * i + 1]);
      }
      // masks: column 2 t of tile j is key t (+ 8 (j & 1) + 16 (j / 2)), column 2 t + 1 is key t + 4
      int lo[2], hi[2], skip[2];                       // a row sees keys [0, skip) and [lo, hi) of the chunk
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (cur.kind == 0) { hi[h] = nvis[h] - cur.at; lo[h] = low[h] - cur.at; skip[h] = min(wr.sinks - cur.at, hi[h]); }
        else { lo[h] = loc[h] - cur.at; hi[h] = nloc[h] == 0x7fffffff ? CHUNK : lo[h] + nloc[h]; skip[h] = 0; }
      }
      const bool whole = hi[0] >= CHUNK && hi[1] >= CHUNK && (lo[0] <= 0 || skip[0] >= CHUNK) && (lo[1] <= 0 || skip[1] >= CHUNK);
      if (!__all_sync(0xffffffffu, whole)) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int h = e >> 1, key = 16 * (j >> 1) + 8 * (j & 1) + t + 4 * (e & 1);
            if (!(key < skip[h] || (key >= lo[h] && key < hi[h]))) s[j][e] = -INFINITY;
          }
      }
      // softmax in base 2; the reference rises only when it is exceeded by the threshold
      uint32_t p[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) mx = sm100::max3(mx, s[j][2 * h], s[j][2 * h + 1]);
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2)) * a.scale_log2;
        const float m_new = mx > m_ref[h] + RAISE_THRESHOLD ? mx : m_ref[h];
        if (__any_sync(0xffffffffu, m_new != m_ref[h])) {
          const float keep = m_new == m_ref[h] ? 1.f : exp2f(m_ref[h] - m_new);
          l_run[h] *= keep;
#pragma unroll
          for (int i = 0; i < NT; ++i) { o[i][2 * h] *= keep; o[i][2 * h + 1] *= keep; }
          m_ref[h] = m_new;
        }
        const float neg = m_ref[h] == -INFINITY ? 0.f : -m_ref[h];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float x = sm100::ex2_approx(fmaf(s[j][2 * h], a.scale_log2, neg)), y = sm100::ex2_approx(fmaf(s[j][2 * h + 1], a.scale_log2, neg));
          l_run[h] += x + y;
          p[j >> 1][2 * (j & 1) + h] = pack_bf16(x, y);
        }
      }
      // P V, eight output tiles at a time
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int k0 = 16 * i + t;                      // the lane's keys: k0, k0 + 4 | k0 + 8, k0 + 12
        uint32_t w[4][NT / 8], ss[2], bb[2];
        if (cur.kind == 0) {
          const uint8_t *codes = vb + g * NT / 32 * L::V_PLANE + g * NT % 32 / 2, *pairs = vb + L::PLANES * L::V_PLANE + g * NT / 32 * 4;
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
        for (int d = 0; d < NT / 8; ++d) {
          uint32_t b[2][8];                             // [pair of keys][dimension]
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t x[4], y[4];                        // the even dimensions of both keys side by side, the odd ones
            if (cur.kind == 0) {
              kv4::values8(__byte_perm(w[2 * h][d], w[2 * h + 1][d], 0x5410), ss[h], bb[h], x);
              kv4::values8(__byte_perm(w[2 * h][d], w[2 * h + 1][d], 0x7632), ss[h], bb[h], y);
            } else {
              const int ka = cur.at + k0 + 8 * h, kc = ka + 4;
              const bf16 *src = a.c.v_local + (long long)seq * wr.k * wr.k * a.c.local_stride + kvh * HD + g * NT + d * 8;
              uint4 u = make_uint4(0, 0, 0, 0), v = u;
              if (ka < wr.k * wr.k) u = *reinterpret_cast<const uint4 *>(src + ka * a.c.local_stride);
              if (kc < wr.k * wr.k) v = *reinterpret_cast<const uint4 *>(src + kc * a.c.local_stride);
              x[0] = __byte_perm(u.x, v.x, 0x5410); x[1] = __byte_perm(u.y, v.y, 0x5410); x[2] = __byte_perm(u.z, v.z, 0x5410); x[3] = __byte_perm(u.w, v.w, 0x5410);
              y[0] = __byte_perm(u.x, v.x, 0x7632); y[1] = __byte_perm(u.y, v.y, 0x7632); y[2] = __byte_perm(u.z, v.z, 0x7632); y[3] = __byte_perm(u.w, v.w, 0x7632);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) { b[h][2 * e] = x[e]; b[h][2 * e + 1] = y[e]; }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) mma(o[8 * d + e], p[i], b[0][e], b[1][e]);
        }
      }
    }

    // ---- the four warps' results: 2 and 3 to 0 and 1, then 1 to 0 ----
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      l_run[h] += __shfl_xor_sync(0xffffffffu, l_run[h], 1);
      l_run[h] += __shfl_xor_sync(0xffffffffu, l_run[h], 2);
    }
    auto hand_over = [&](int area) {
      float *x = reinterpret_cast<float *>(few_smem + L::MERGE_OFF + area * L::MERGE_BYTES) + lane;
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[(4 * i + e) * 32] = o[i][e];
      x[(L::O_REGS + 0) * 32] = m_ref[0]; x[(L::O_REGS + 1) * 32] = m_ref[1]; x[(L::O_REGS + 2) * 32] = l_run[0]; x[(L::O_REGS + 3) * 32] = l_run[1];
    };
    auto take_over = [&](int area) {
      const float *x = reinterpret_cast<const float *>(few_smem + L::MERGE_OFF + area * L::MERGE_BYTES) + lane;
      float mine_w[2], other_w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float other = x[(L::O_REGS + h) * 32], M = fmaxf(m_ref[h], other);
        mine_w[h] = m_ref[h] == -INFINITY ? 0.f : exp2f(m_ref[h] - M); other_w[h] = other == -INFINITY ? 0.f : exp2f(other - M);
        l_run[h] = mine_w[h] * l_run[h] + other_w[h] * x[(L::O_REGS + 2 + h) * 32];
        m_ref[h] = M;
      }
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] = mine_w[e >> 1] * o[i][e] + other_w[e >> 1] * x[(4 * i + e) * 32];
    };
    static_assert(NT * 4 == L::O_REGS, "a warp's O");
    if (warp >= 2) hand_over(warp - 2);
    __syncthreads();
    if (warp < 2) take_over(warp);
    if (warp == 1) hand_over(2);
    __syncthreads();
    const bool cut = u0 < w0 || u1 > w1;
    const int first_cta = cut ? (int)(((u0 + 1) * C - 1) / W) : 0, last_cta = cut ? (int)((u1 * C - 1) / W) : 0;      // shares that the unit's first and last chunk lie in
    if (warp == 0) {
      take_over(2);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = g + 8 * h, m = tile * ROWS + r, slot = m / G;
        if (r >= rows_here) continue;
        if (!cut) {
          const float inv = l_run[h] > 0.f ? 1.f / l_run[h] : 0.f;         // (a row that sees nothing: zeros)
          bf16 *dst = a.c.out + (((long long)seq * T + slot) * a.c.Hq + kvh * G + (m - slot * G)) * HD;
#pragma unroll
          for (int run = 0; run < 2; ++run)                                // dimensions (2 t + run) NT .. + NT
#pragma unroll
            for (int d = 0; d < NT; d += 8) {
              uint4 u;
              u.x = pack_bf16(o[d][2 * h + run] * inv, o[d + 1][2 * h + run] * inv); u.y = pack_bf16(o[d + 2][2 * h + run] * inv, o[d + 3][2 * h + run] * inv);
              u.z = pack_bf16(o[d + 4][2 * h + run] * inv, o[d + 5][2 * h + run] * inv); u.w = pack_bf16(o[d + 6][2 * h + run] * inv, o[d + 7][2 * h + run] * inv);
              *reinterpret_cast<uint4 *>(dst + (2 * t + run) * NT + d) = u;
            }
        } else {
          const size_t part = (size_t)(2 * blockIdx.x + (u0 >= w0)) * ROWS + r;
          float *dst = a.part_O + part * HD;
#pragma unroll
          for (int run = 0; run < 2; ++run)
#pragma unroll
            for (int d = 0; d < NT; d += 4)
              *reinterpret_cast<float4 *>(dst + (2 * t + run) * NT + d) = make_float4(o[d][2 * h + run], o[d + 1][2 * h + run], o[d + 2][2 * h + run], o[d + 3][2 * h + run]);
          if (t == 0) a.part_ml[part] = make_float2(m_ref[h], l_run[h]);
        }
      }
      if (cut) {
        __threadfence();
        __syncwarp();
        if (lane == 0) is_last = atomicAdd(&a.arrived[first_cta], 1) == last_cta - first_cta;
      }
    }
    if (cut) {
      __syncthreads();
      if (is_last) {
        __threadfence();
        const int pieces = last_cta - first_cta + 1;
        for (int i = threadIdx.x; i < rows_here * (HD / 4); i += WARPS * 32) {
          const int r = i / (HD / 4), d = i % (HD / 4) * 4;
          auto part = [&](int x) { return (size_t)(2 * (first_cta + x) + (x == 0)) * ROWS + r; };
          float M = -INFINITY, den = 0.f;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int x0 = 0; x0 < pieces; x0 += 4) {      // four at a time, their loads ahead of the first use
            float2 ml[4]; float4 v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              ml[e] = make_float2(-INFINITY, 0.f); v[e] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (x0 + e < pieces) { ml[e] = __ldcg(a.part_ml + part(x0 + e)); v[e] = __ldcg(reinterpret_cast<const float4 *>(a.part_O + part(x0 + e) * HD + d)); }
            }
            const float top = fmaxf(fmaxf(M, fmaxf(ml[0].x, ml[1].x)), fmaxf(ml[2].x, ml[3].x));
            const float keep = M == -INFINITY ? 0.f : exp2f(M - top);
            M = top; den *= keep;
            acc.x *= keep; acc.y *= keep; acc.z *= keep; acc.w *= keep;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float w = ml[e].x == -INFINITY ? 0.f : exp2f(ml[e].x - M);
              den += w * ml[e].y;
              acc.x = fmaf(w, v[e].x, acc.x); acc.y = fmaf(w, v[e].y, acc.y); acc.z = fmaf(w, v[e].z, acc.z); acc.w = fmaf(w, v[e].w, acc.w);
            }
          }
          const float inv = den > 0.f ? 1.f / den : 0.f;
          const int m = tile * ROWS + r, slot = m / G;
          uint2 u;
          u.x = pack_bf16(acc.x * inv, acc.y * inv); u.y = pack_bf16(acc.z * inv, acc.w * inv);
          *reinterpret_cast<uint2 *>(a.c.out + (((long long)seq * T + slot) * a.c.Hq + kvh * G + (m - slot * G)) * HD + d) = u;
        }
        if (threadIdx.x == 0) a.arrived[first_cta] = 0;
      }
    }
    a0 = a1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

}  // namespace attn_few
