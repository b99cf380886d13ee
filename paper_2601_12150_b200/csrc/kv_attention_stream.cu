// Attention of few query rows over the 8-bit cache: the step of a decoder.
//
// Bound by HBM: 2 * head_dim bytes a key and key head are read once, for 4 * head_dim * rows operations.
//
//   kv_stream_kernel  one CTA per SM.  All key tiles (8 KB) of all (sequence, key head) pairs form one line,
//                     and every CTA takes an equal stretch of it, whatever the lengths are.  A producer warp brings
//                     the tiles in by TMA (as many in flight as shared memory holds: the latency of HBM times its
//                     rate is 35 KB an SM); the other warps take them in turn, each with an online softmax of its own,
//                     and join their states where the pair changes.  Codes go from shared memory to fp16 fragments
//                     in registers (the 128-byte swizzle makes the 16-byte reads of both operands free of bank
//                     conflicts), and the products run with keys as the rows: S^T = K Q^T and O^T = V^T P^T, so
//                     that eight queries fill the narrow side of mma.m16n8k16 and P^T comes out of the score
//                     fragments with one 8 x 8 transpose.
//   kv_finish_kernel  joins the pieces of pairs that were cut between CTAs, and turns the stored scores into
//                     attention weights.
//
// Numbers: queries are scaled by a power of two of their own (largest magnitude in [2^14, 2^15)) into fp16, exactly but
// for elements below 2^-28 of their row's largest; codes are exact in fp16; sums are fp32.  Probabilities are rounded to
// fp16 for the product with V (relative 2^-11, less than the rounding of the result to bf16) and relative to a maximum
// that is renewed only when a score exceeds it by more than 2^8; the denominator sums them unrounded.
#include "kv_attention.cuh"

namespace {

using namespace spv;

// slots of a key tile: 8 KB of keys and values
__host__ __device__ constexpr int tile_of(int head_dim) { return head_dim == 128 ? 32 : 64; }
constexpr int kMergeWarps = 8;               // warps whose results are added up at a time
constexpr int kPartSlots = 2;                // pieces a CTA can leave: of the pair it began in, of the one it ended in
constexpr float kLazy = 8.0f;
constexpr int kIssue = 4;                    // tiles that the producer's lanes bring in side by side

struct StreamArgs {
  KvAttnArgs a;
  float* z;             // scores (log2 domain) [tile][rows][slot], NULL when no weights are wanted
  float* part_o;        // [CTA][2][8 NT][D] unnormalised
  float2* part_ml;      // [CTA][2][8 NT] maximum, sum
  float2* pair_ml;      // [pair][8 NT]: the same of pairs that one CTA had whole
  int32_t rows;         // tokens * group
};

struct StageMeta {      // of one tile, by 16-slot quarters
  float ks[4], vs[4];
  int bad;              // bit i: quarter i names no page
  int pad[3];
};

template <int D, int NT>
struct Layout {
  // place of tile `it` of the CTA, and the phase of that stage's barriers
  __device__ static int stage(uint32_t it) { return (int)(it % kWarps * kOwn + it / kWarps % kOwn); }
  __device__ static uint32_t phase(uint32_t it) { return it / kWarps / kOwn; }
  static constexpr int kTile = tile_of(D);
  // consumer warps: with the producer 3 or 2 a scheduler, which leaves 168 or 255 registers a thread
  static constexpr int kWarps = NT < 4 ? 11 : 7;
  static constexpr int kThreads = (kWarps + 1) * 32;
  static constexpr int kStageBytes = 2 * kTile * D;
  static constexpr int kMergePitch = D + 4;
  static constexpr int kMerge = kMergeWarps * 8 * kMergePitch * 4;
  static constexpr int kQ = NT * (D / 16) * 32 * 8;
  static constexpr int kRows = 8 * NT;
  static constexpr int kSmall = kRows * 4 * 2 + kWarps * kRows * 8 + 2048;
  static constexpr int kBudget = 227 * 1024 - 1024;
  static constexpr int kFit = (kBudget - kMerge - kQ - kSmall) / (kStageBytes + (int)sizeof(StageMeta) + 16);
  // Stages belong to one consumer warp each, which waits for their phases one after the other: a parity says which of
  // two phases is over, so nobody may wait for a phase while the one before it is still to come.
  static constexpr int kOwn = kFit / kWarps;
  static constexpr int kStages = kOwn * kWarps;
  static constexpr int oMerge = kStages * kStageBytes;
  static constexpr int oQ = oMerge + kMerge;
  static constexpr int oMeta = oQ + kQ;
  static constexpr int oBars = oMeta + kStages * (int)sizeof(StageMeta);
  static constexpr int oEnd = oBars + kStages * 16;
  static constexpr int oFactor = oEnd + kRows * 4;
  static constexpr int oMl = oFactor + kRows * 4;                       // float2 [warp][row]
  static constexpr int oScan = oMl + kWarps * kRows * 8;
  static constexpr int kTotal = oScan + 512;
};

// ---- the line of tiles -------------------------------------------------------------------------
struct Scan {
  int64_t total, before;     // tiles of all sequences; of those before the one that holds the target
  int64_t warp_sum[16];
  int b;
};

__device__ __forceinline__ int seq_len(const KvView& c, int b) { return spv_kv_clamp(__ldg(c.lengths + b), c.max_length); }
__device__ __forceinline__ int seq_queries(const KvAttnArgs& a, int b) {
  return a.counts ? spv_kv_clamp(__ldg(a.counts + b), a.tokens) : a.tokens;
}
template <int TILE>
__device__ __forceinline__ int seq_key_tiles(const KvView& c, const KvAttnArgs& a, int b) {
  return seq_queries(a, b) > 0 ? (seq_len(c, b) + TILE - 1) / TILE : 0;
}

// Sums the tiles of all sequences; then the sequence that holds tile `share(total)`.  All threads of the CTA.
template <int THREADS, int TILE, typename F>
__device__ __forceinline__ void scan_tiles(const KvView& c, const KvAttnArgs& a, Scan* s, F share) {
  const int per = (a.batch + THREADS - 1) / THREADS;
  const int b0 = threadIdx.x * per, b1 = min(a.batch, b0 + per);
  int64_t sum = 0;
  for (int b = b0; b < b1; ++b) sum += (int64_t)c.kv_heads * seq_key_tiles<TILE>(c, a, b);
  int64_t inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, inc, o);
    if ((threadIdx.x & 31) >= o) inc += x;
  }
  if ((threadIdx.x & 31) == 31) s->warp_sum[threadIdx.x >> 5] = inc;
  __syncthreads();
  int64_t base = 0, total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < (threadIdx.x >> 5)) base += s->warp_sum[w];
    total += s->warp_sum[w];
  }
  const int64_t target = share(total);
  int64_t at = base + inc - sum;
  if (target >= at && target < at + sum) {
    int b = b0;
    for (;; ++b) {
      const int64_t t = (int64_t)c.kv_heads * seq_key_tiles<TILE>(c, a, b);
      if (target < at + t || b + 1 >= b1) break;
      at += t;
    }
    s->b = b;
    s->before = at;
  }
  if (threadIdx.x == 0) s->total = total;
  __syncthreads();
}

// CTAs that get a stretch: every one of them has a tile at least, so that no piece between two others is missing.
__device__ __forceinline__ int working_ctas(int64_t total, int ctas) { return (int)min(total, (int64_t)ctas); }
__device__ __forceinline__ int64_t stretch_begin(int64_t total, int cta, int ctas) { return total * cta / ctas; }
// the CTA whose stretch holds tile t
__device__ __forceinline__ int tile_owner(int64_t total, int64_t t, int ctas) { return (int)(((t + 1) * ctas - 1) / total); }

// One piece of a pair: key tiles [kt0, kt1) of `tiles`.
struct Piece {
  int b, head, len, n, tiles, kt0, kt1;
  int64_t line;              // place of kt0 on the line
};
struct Walk {
  int64_t pos, end, before;
  int b;
};
template <int TILE>
__device__ __forceinline__ bool next_piece(const KvView& c, const KvAttnArgs& a, Walk& w, Piece& p) {
  if (w.pos >= w.end) return false;
  int tiles = seq_key_tiles<TILE>(c, a, w.b);
  while (w.pos >= w.before + (int64_t)c.kv_heads * tiles) {
    w.before += (int64_t)c.kv_heads * tiles;
    if (++w.b >= a.batch) return false;
    tiles = seq_key_tiles<TILE>(c, a, w.b);
  }
  const int off = (int)(w.pos - w.before);
  p.b = w.b;
  p.head = off / tiles;
  p.kt0 = off % tiles;
  p.kt1 = (int)min((int64_t)tiles, p.kt0 + (w.end - w.pos));
  p.tiles = tiles;
  p.len = seq_len(c, w.b);
  p.n = seq_queries(a, w.b);
  p.line = w.pos;
  w.pos += p.kt1 - p.kt0;
  return true;
}

// ---- pieces of the consumer ----------------------------------------------------------------------
__device__ __forceinline__ void tma_load_rows(void* dst, const CUtensorMap* m, uint64_t* bar, int row, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%3, %4}], [%2], %5;" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(0), "r"(row), "l"(policy)
      : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}

// Queries of a pair to shared memory in fragment order: [query tile][k step][lane][4], lane = 4 * query + c, the four
// values d = (D/4) c + 4 step .. + 3.  Rows behind the last are zeros.
template <int D, int NT>
__device__ __forceinline__ void load_queries(const StreamArgs& s, const Piece& p, uint16_t* q, float* factor, int* ends) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kPer = D / 32;     // elements of a row for each lane
  for (int row = warp; row < 8 * NT; row += Layout<D, NT>::kWarps) {
    const int i = row / s.a.group, head = p.head * s.a.group + row % s.a.group;
    float x[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] = 0.0f;
    const bool real = i < p.n;
    if (real) {
      const uint16_t* src = s.a.q + p.b * s.a.q_stride_b + i * s.a.q_stride_tok + head * s.a.q_stride_head + lane * kPer;
      uint32_t w[kPer / 2];
#pragma unroll
      for (int e = 0; e < kPer / 2; ++e) w[e] = __ldg(reinterpret_cast<const uint32_t*>(src) + e);
#pragma unroll
      for (int e = 0; e < kPer / 2; ++e) {
        const float2 f = s.a.dtype == SPV_BF16 ? kv_unpack2<SPV_BF16>(w[e]) : kv_unpack2<SPV_FP16>(w[e]);
        x[2 * e] = f.x;
        x[2 * e + 1] = f.y;
      }
    }
    uint32_t big = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) big = max(big, __float_as_uint(x[e]) & 0x7FFFFFFFu);
    big = __reduce_max_sync(0xffffffffu, big);
    const int ex = max((int)(big >> 23) - 127, -100);
    const float up = kv_pow2(14 - ex);
#pragma unroll
    for (int e = 0; e < kPer; e += 2) {
      const __half2 h = __floats2half2_rn(x[e] * up, x[e + 1] * up);
      const int d = lane * kPer + e, c = d / (D / 4), step = d % (D / 4) / 4;
      const int at = (((row >> 3) * (D / 16) + step) * 32 + (row & 7) * 4 + c) * 4 + (d & 3);
      *reinterpret_cast<__half2*>(q + at) = h;
    }
    if (lane == 0) {
      factor[row] = s.a.scale * 1.4426950408889634f * kv_pow2(ex - 14);
      ends[row] = real ? spv_kv_query_end(p.len, p.n, i, s.a.causal) : p.len;
    }
  }
}

template <int FMT, int D, int NT>
__global__ void __launch_bounds__(Layout<D, NT>::kThreads, 1)
    kv_stream_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const KvView c,
                     const StreamArgs s) {
  using L = Layout<D, NT>;
  constexpr int kRows = L::kRows;
  constexpr int kWarps = L::kWarps;
  constexpr int kTile = L::kTile;
  constexpr int kQuarters = kTile / 16;        // scales are kept for 16 slots each
  constexpr int kSteps = D / 16;             // k steps of S^T, row tiles of O^T
  constexpr int kKeys = NT < 4 || D == 64 ? 32 : 16;   // keys whose scores are held at once
  constexpr int kMt = kKeys / 16;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  float* merge = reinterpret_cast<float*>(smem + L::oMerge);
  uint16_t* sq = reinterpret_cast<uint16_t*>(smem + L::oQ);
  StageMeta* meta = reinterpret_cast<StageMeta*>(smem + L::oMeta);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::oBars);
  uint64_t* empty = full + L::kStages;
  int* ends = reinterpret_cast<int*>(smem + L::oEnd);
  float* factor = reinterpret_cast<float*>(smem + L::oFactor);
  float2* sml = reinterpret_cast<float2*>(smem + L::oMl);
  Scan* scan = reinterpret_cast<Scan*>(smem + L::oScan);
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem + L::oScan + 256);
  uint32_t* wait_status = c.status - 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
    for (int i = 0; i < L::kStages; ++i) {
      mbar_init(full + i, 2);
      mbar_init(empty + i, 1);
    }
    mbar_fence_init();
    *abort_flag = 0u;
  }
  if (blockIdx.x == 0) {       // the caller's numbers: a bad one is latched once
    for (int b = threadIdx.x; b < s.a.batch; b += L::kThreads) {
      kv_clamped(__ldg(c.lengths + b), c.max_length, c.status);
      if (s.a.counts) kv_clamped(__ldg(s.a.counts + b), s.a.tokens, c.status);
    }
  }
  scan_tiles<L::kThreads, kTile>(c, s.a, scan, [&](int64_t total) {
    const int w = working_ctas(total, gridDim.x);
    return blockIdx.x < w ? stretch_begin(total, blockIdx.x, w) : total;
  });
  asm volatile("griddepcontrol.launch_dependents;");
  const int64_t total = scan->total;
  const int working = working_ctas(total, gridDim.x);
  if (blockIdx.x >= working) return;
  Walk walk;
  walk.pos = stretch_begin(total, blockIdx.x, working);
  walk.end = stretch_begin(total, blockIdx.x + 1, working);
  walk.before = scan->before;
  walk.b = scan->b;
  Piece p;

  if (warp == kWarps) {
    // ---- producer: every lane has a tile of its own, and kIssue lanes at a time wait, copy and describe; the page
    // numbers of the next 32 tiles are on their way meanwhile
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    const int part = min(s.a.block, kTile);              // slots that one copy brings
    const int parts = kTile / part;                      // copies of a tile: 1, 2 or 4
    uint32_t it = 0;
    while (next_piece<kTile>(c, s.a, walk, p)) {
      const int32_t* row = c.table + p.b * c.table_stride;
      int next[kQuarters];
      auto fetch = [&](int kt) {
#pragma unroll
        for (int x = 0; x < kQuarters; ++x) {
          const int slot = kt * kTile + x * part;
          next[x] = x < parts && kt < p.kt1 && slot < p.len ? __ldg(row + slot / s.a.block) : INT32_MIN;
        }
      };
      fetch(p.kt0 + lane);
      for (int base = p.kt0; base < p.kt1; base += 32) {
        const int kt = base + lane;
        int page[kQuarters];
        float ks[kQuarters], vs[kQuarters];
        int loads = 0, bad = 0;
#pragma unroll
        for (int x = 0; x < kQuarters; ++x) {
          page[x] = next[x];
          ks[x] = vs[x] = 0.0f;                          // of parts that hold nothing
          if (spv_kv_valid_page(page[x], c.pages)) {
            const size_t ph = (size_t)page[x] * c.kv_heads + p.head;
            ks[x] = __ldg(c.k_scale + ph);
            vs[x] = __ldg(c.v_scale + ph);
            ++loads;
          } else if (x < parts && kt < p.kt1 && kt * kTile + x * part < p.len) {
            kv_fault(c.status, SPV_SITE_KV_PAGE);
            bad |= ((1 << kQuarters / parts) - 1) << x * (kQuarters / parts);
          }
        }
        if (base + 32 < p.kt1) fetch(base + 32 + lane);
        const int count = min(32, p.kt1 - base);
        for (int j = 0; j < count; j += kIssue) {
          if (lane >= j && lane < min(j + kIssue, count)) {
            const uint32_t at = it + lane;
            const int st = L::stage(at);
            if (at >= L::kStages) mbar_wait(empty + st, (L::phase(at) - 1) & 1, abort_flag, wait_status, 0x4B01u);
            uint8_t* kdst = smem + st * L::kStageBytes;
            mbar_expect_tx(full + st, loads * 2 * part * D);
#pragma unroll
            for (int x = 0; x < kQuarters; ++x) {
              if (spv_kv_valid_page(page[x], c.pages)) {
                const int at_row = (int)(spv_kv_row(page[x], c.kv_heads, p.head, s.a.block, kt * kTile + x * part) / (128 / D));
                tma_load_rows(kdst + x * part * D, &map_k, full + st, at_row, policy);
                tma_load_rows(kdst + kTile * D + x * part * D, &map_v, full + st, at_row, policy);
              }
            }
            StageMeta* m = meta + st;
#pragma unroll
            for (int x = 0; x < kQuarters; ++x) {
              const int y = x * parts / kQuarters;       // part that quarter x is in
              float kx = ks[0], vx = vs[0];
#pragma unroll
              for (int i = 1; i < kQuarters; ++i) {
                kx = y == i ? ks[i] : kx;
                vx = y == i ? vs[i] : vx;
              }
              m->ks[x] = kx;
              m->vs[x] = vx;
            }
            m->bad = bad;
            mbar_arrive(full + st);
          }
          __syncwarp();
        }
        it += count;
      }
    }
    // nothing of this CTA is in flight when it ends: a wait that gave up leaves copies behind
    if (*abort_flag != 0u && lane == 0) {
      for (uint32_t i = it > L::kStages ? it - L::kStages : 0; i < it; ++i)
        for (int tries = 0; tries < 1000 && !mbar_try_wait_parked(full + L::stage(i), L::phase(i) & 1, 1000u); ++tries) {
        }
    }
    return;
  }

  // ---- consumers
  const int r = lane >> 2, q2 = (lane & 3) * 2;
  uint32_t ring = 0;
  while (next_piece<kTile>(c, s.a, walk, p)) {
    load_queries<D, NT>(s, p, sq, factor, ends);
    asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
    const int full_end = ends[0];           // slots that every query sees (row 0 sees least)
    float o[kSteps][NT][4];
    float m[NT][2], l[NT][2], qf[NT][2];
    float vref = 0.0f, vtop = 0.0f;         // unit of o; largest value scale met
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[t][e] = -INFINITY;
        l[t][e] = 0.0f;
        qf[t][e] = factor[8 * t + q2 + e];
      }
#pragma unroll
      for (int j = 0; j < kSteps; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][t][e] = 0.0f;
    }
    uint2 qr[NT == 1 ? kSteps : 1];
    const uint32_t sq_at = smem_u32(sq) + lane * 8;
    if (NT == 1) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) qr[NT == 1 ? j : 0] = lds64(sq_at + j * 256);
    }
    const uint32_t ring_end = ring + (p.kt1 - p.kt0);
    for (uint32_t it = ring + (warp + kWarps - ring % kWarps) % kWarps; it < ring_end; it += kWarps) {
      const int st = L::stage(it);
      const int kt = p.kt0 + (int)(it - ring);
      mbar_wait(full + st, L::phase(it) & 1, abort_flag, wait_status, 0x4B02u);
      const uint32_t kbase = smem_u32(smem) + st * L::kStageBytes, vbase = kbase + kTile * D;
      const StageMeta* mt_at = meta + st;
      const int bad = mt_at->bad;
      const bool edge = (kt + 1) * kTile > full_end || bad != 0;
      // the unit of o follows the value scales by powers of two and more, not by every block's own
      float vt = mt_at->vs[0];
#pragma unroll
      for (int x = 1; x < kQuarters; ++x) vt = fmaxf(vt, mt_at->vs[x]);
      vtop = fmaxf(vtop, vt);
      if (!(vt <= vref * 16.0f && vt >= vref * 0.0625f)) {
        const float next = fmaxf(vt, vtop * 0x1p-60f);
        const float f = vref > 0.0f ? vref / next : 0.0f;
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[j][t][e] *= f;
        vref = next;
      }
      const float vinv = vref > 0.0f ? 1.0f / vref : 0.0f;
#pragma unroll 1     // the body once: several warps a scheduler at different places of it share its instruction cache
      for (int half = 0; half < kTile / kKeys; ++half) {
        float z[kMt][NT][4];
#pragma unroll
        for (int i = 0; i < kMt; ++i) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) z[i][t][e] = 0.0f;
          const int key = half * kKeys + i * 16 + r;
          uint32_t wa[kSteps], wb[kSteps];
          if (D == 128) {
            const uint32_t at = kbase + key * 128;
            const uint32_t c0 = ((q2 ^ r) << 4), c1 = (((q2 + 1) ^ r) << 4);
            *reinterpret_cast<uint4*>(wa) = lds128(at + c0);
            *reinterpret_cast<uint4*>(wa + 4) = lds128(at + c1);
            *reinterpret_cast<uint4*>(wb) = lds128(at + 1024 + c0);
            *reinterpret_cast<uint4*>(wb + 4) = lds128(at + 1024 + c1);
          } else {
            const int line = key >> 1, chunk = (key & 1) * 4 + (lane & 3);
            *reinterpret_cast<uint4*>(wa) = lds128(kbase + line * 128 + ((chunk ^ (line & 7)) << 4));
            *reinterpret_cast<uint4*>(wb) = lds128(kbase + (line + 4) * 128 + ((chunk ^ ((line + 4) & 7)) << 4));
          }
#pragma unroll
          for (int j = 0; j < kSteps; ++j) {
            uint32_t a0, a1, a2, a3;
            kv_half4<FMT>(wa[j], a0, a2);
            kv_half4<FMT>(wb[j], a1, a3);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              const uint2 b = NT == 1 ? qr[NT == 1 ? j : 0] : lds64(sq_at + (t * kSteps + j) * 256);
              mma_16816(z[i][t], a0, a1, a2, a3, b.x, b.y);
            }
          }
        }
        // scores in the log2 domain, masked
#pragma unroll
        for (int i = 0; i < kMt; ++i) {
          const float ks = mt_at->ks[half * (kKeys / 16) + i];
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) z[i][t][e] *= ks * qf[t][e & 1];
        }
        if (edge) {
#pragma unroll
          for (int i = 0; i < kMt; ++i) {
            const int quarter = half * (kKeys / 16) + i;
            const int slot = kt * kTile + quarter * 16 + r;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (slot + (e >> 1) * 8 >= ends[8 * t + q2 + (e & 1)] || (bad >> quarter & 1)) z[i][t][e] = -INFINITY;
          }
        }
        if (s.z) {
          float* zt = s.z + (size_t)(p.line + (kt - p.kt0)) * s.rows * kTile;
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int row = 8 * t + q2 + e;
              if (row < s.rows) {
#pragma unroll
                for (int i = 0; i < kMt; ++i) {
                  float* at = zt + row * kTile + half * kKeys + i * 16 + r;
                  at[0] = z[i][t][e];
                  at[8] = z[i][t][e + 2];
                }
              }
            }
        }
        // running maxima: renewed for all when any score is far above its own
        float top[NT][2];
        bool above = false;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            top[t][e] = z[0][t][e];
#pragma unroll
            for (int i = 0; i < kMt; ++i) top[t][e] = fmaxf(top[t][e], fmaxf(z[i][t][e], z[i][t][e + 2]));
            above |= top[t][e] > m[t][e] + kLazy;
          }
        if (__any_sync(0xffffffffu, above)) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float x = fmaxf(top[t][e], m[t][e]);
#pragma unroll
              for (int sh = 4; sh < 32; sh <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, sh));
              const float f = exp2_fast(m[t][e] - (x == -INFINITY ? 0.0f : x));
              m[t][e] = x;
              l[t][e] *= f;
#pragma unroll
              for (int j = 0; j < kSteps; ++j) {
                o[j][t][e] *= f;
                o[j][t][e + 2] *= f;
              }
            }
        }
        uint32_t pb[kMt][NT][2];
#pragma unroll
        for (int i = 0; i < kMt; ++i) {
          const float vr = mt_at->vs[half * (kKeys / 16) + i] * vinv;
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float mm = m[t][e & 1];
              x[e] = exp2_fast(z[i][t][e] - (mm == -INFINITY ? 0.0f : mm));
              l[t][e & 1] += x[e];
              x[e] *= vr;
            }
            pb[i][t][0] = transpose_8x8(kv_pack2<SPV_FP16>(x[0], x[1]));
            pb[i][t][1] = transpose_8x8(kv_pack2<SPV_FP16>(x[2], x[3]));
          }
        }
        // O^T += V^T P^T, 16 keys at a time
#pragma unroll
        for (int i = 0; i < kMt; ++i) {
          constexpr int kW = D / 32;                    // words of a key's row for each thread
          uint32_t w[4][kW];
          const int key0 = half * kKeys + i * 16 + q2;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int key = key0 + (x & 1) + (x >> 1) * 8;
            if (D == 128) {
              *reinterpret_cast<uint4*>(w[x]) = lds128(vbase + key * 128 + ((r ^ (key & 7)) << 4));
            } else {
              const int line = key >> 1, chunk = (key & 1) * 4 + (r >> 1);
              *reinterpret_cast<uint2*>(w[x]) = lds64(vbase + line * 128 + ((chunk ^ (line & 7)) << 4) + (r & 1) * 8);
            }
          }
          if (edge) {   // what lies behind the last token may be any bits, NaN among them
            const int quarter = half * (kKeys / 16) + i;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int slot = kt * kTile + key0 + (x & 1) + (x >> 1) * 8;
              if (slot >= p.len || (bad >> quarter & 1)) {
#pragma unroll
                for (int y = 0; y < kW; ++y) w[x][y] = 0u;
              }
            }
          }
#pragma unroll
          for (int y = 0; y < kW; ++y) {
            uint32_t a[2][4];     // row tiles 2y and 2y + 1
#pragma unroll
            for (int x = 0; x < 2; ++x) {       // keys 2c, 2c+1 and 2c+8, 2c+9
              uint32_t h[4];
              kv_half4<FMT>(__byte_perm(w[2 * x][y], w[2 * x + 1][y], 0x5140), h[0], h[1]);
              kv_half4<FMT>(__byte_perm(w[2 * x][y], w[2 * x + 1][y], 0x7362), h[2], h[3]);
              a[0][2 * x] = h[0];
              a[0][2 * x + 1] = h[1];
              a[1][2 * x] = h[2];
              a[1][2 * x + 1] = h[3];
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              mma_16816(o[2 * y][t], a[0][0], a[0][1], a[0][2], a[0][3], pb[i][t][0], pb[i][t][1]);
              mma_16816(o[2 * y + 1][t], a[1][0], a[1][1], a[1][2], a[1][3], pb[i][t][0], pb[i][t][1]);
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty + st);
    }
    ring = ring_end;

    // ---- the warps' states into one
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int sh = 4; sh < 32; sh <<= 1) l[t][e] += __shfl_xor_sync(0xffffffffu, l[t][e], sh);
        if (r == 0) sml[warp * kRows + 8 * t + q2 + e] = make_float2(m[t][e], l[t][e]);
      }
    asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
    const bool whole = p.kt0 == 0 && p.kt1 == p.tiles;
    const int slot = 2 * blockIdx.x + (p.kt0 > 0 ? 0 : 1);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      constexpr int kParts = 8 * (D / 4);                              // float4s of eight queries' rows
      constexpr int kMine = (kParts + kWarps * 32 - 1) / (kWarps * 32);
      float4 sums[kMine];
#pragma unroll
      for (int y = 0; y < kMine; ++y) sums[y] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int w0 = 0; w0 < kWarps; w0 += kMergeWarps) {
        if (w0 <= warp && warp < w0 + kMergeWarps) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sml[w * kRows + 8 * t + q2 + e].x);
            const float f = m[t][e] == -INFINITY ? 0.0f : exp2_fast(m[t][e] - top) * vref;
            float* at = merge + ((warp - w0) * 8 + q2 + e) * L::kMergePitch + r * (D / 8);
#pragma unroll
            for (int j = 0; j < kSteps; j += 2)
              *reinterpret_cast<float4*>(at + 2 * j) =
                  make_float4(o[j][t][e] * f, o[j][t][e + 2] * f, o[j + 1][t][e] * f, o[j + 1][t][e + 2] * f);
          }
        }
        asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
#pragma unroll
        for (int y = 0; y < kMine; ++y) {
          const int x = threadIdx.x + y * kWarps * 32;
          if (x < kParts) {
            const float* at = merge + x / (D / 4) * L::kMergePitch + x % (D / 4) * 4;
#pragma unroll
            for (int w = w0; w < kWarps && w < w0 + kMergeWarps; ++w) {
              const float4 v = *reinterpret_cast<const float4*>(at + (w - w0) * 8 * L::kMergePitch);
              sums[y].x += v.x;
              sums[y].y += v.y;
              sums[y].z += v.z;
              sums[y].w += v.w;
            }
          }
        }
        asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");
      }
#pragma unroll
      for (int y = 0; y < kMine; ++y) {
        const int x = threadIdx.x + y * kWarps * 32;
        if (x >= kParts) continue;
        const float4 sum = sums[y];
        const int qi = x / (D / 4), d = x % (D / 4) * 4, row = 8 * t + qi;
        float top = -INFINITY, den = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sml[w * kRows + row].x);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float2 ml = sml[w * kRows + row];
          den += ml.x == -INFINITY ? 0.0f : ml.y * exp2_fast(ml.x - top);
        }
        if (whole) {
          const int i = row / s.a.group, head = p.head * s.a.group + row % s.a.group;
          if (i < p.n) {
            const float inv = top == -INFINITY ? 0.0f : 1.0f / den;
            uint16_t* out = s.a.o + p.b * s.a.o_stride_b + i * s.a.o_stride_tok + head * s.a.o_stride_head + d;
            uint2 u;
            if (s.a.dtype == SPV_BF16) {
              u.x = kv_pack2<SPV_BF16>(sum.x * inv, sum.y * inv);
              u.y = kv_pack2<SPV_BF16>(sum.z * inv, sum.w * inv);
            } else {
              u.x = kv_pack2<SPV_FP16>(sum.x * inv, sum.y * inv);
              u.y = kv_pack2<SPV_FP16>(sum.z * inv, sum.w * inv);
            }
            *reinterpret_cast<uint2*>(out) = u;
            if (d == 0) {
              if (s.a.lse)
                s.a.lse[((size_t)p.b * s.a.tokens + i) * s.a.heads + head] =
                    top == -INFINITY ? -INFINITY : (top + log2f(den)) * 0.6931471805599453f;
              s.pair_ml[(size_t)(p.b * c.kv_heads + p.head) * kRows + row] = make_float2(top, den);
            }
          }
        } else {
          *reinterpret_cast<float4*>(s.part_o + ((size_t)slot * kRows + row) * D + d) = sum;
          if (d == 0) s.part_ml[(size_t)slot * kRows + row] = make_float2(top, den);
        }
      }
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory");     // sml is read no more
  }
}

// ---- pieces and weights --------------------------------------------------------------------------
constexpr int kFinishThreads = 256;
constexpr int kFinishKeys = 1024;

// grid (parts of the slots, key heads * batch); the first part also joins the pieces
template <int D>
__global__ void __launch_bounds__(kFinishThreads) kv_finish_kernel(const KvView c, const StreamArgs s, int ctas, int row_slots) {
  constexpr int kTile = tile_of(D);
  __shared__ float2 stat[kKvStreamMaxRows];       // maximum, 1 / sum of a row
  const int pair = blockIdx.y, b = pair / c.kv_heads, head = pair % c.kv_heads;
  const int len = seq_len(c, b), n = seq_queries(s.a, b), rows = n * s.a.group;
  const int key0 = blockIdx.x * kFinishKeys;
  const bool weights = s.a.w_out != nullptr && key0 < len;
  // tiles before this sequence: those of the sequences 0 .. b - 1
  int64_t before = 0, all = 0;
  for (int i = threadIdx.x; i < s.a.batch; i += kFinishThreads) {
    const int64_t t = (int64_t)c.kv_heads * seq_key_tiles<kTile>(c, s.a, i);
    all += t;
    if (i < b) before += t;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    before += __shfl_xor_sync(0xffffffffu, before, o);
    all += __shfl_xor_sync(0xffffffffu, all, o);
  }
  __shared__ int64_t sums[kFinishThreads / 32][2];
  if ((threadIdx.x & 31) == 0) { sums[threadIdx.x >> 5][0] = before; sums[threadIdx.x >> 5][1] = all; }
  __syncthreads();
  before = all = 0;
#pragma unroll
  for (int w = 0; w < kFinishThreads / 32; ++w) { before += sums[w][0]; all += sums[w][1]; }
  const int tiles = seq_key_tiles<kTile>(c, s.a, b);
  const int64_t line = before + (int64_t)head * tiles;
  const int working = working_ctas(all, ctas);
  const int c0 = tiles ? tile_owner(all, line, working) : 0, c1 = tiles ? tile_owner(all, line + tiles - 1, working) : 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (weights || (blockIdx.x == 0 && c0 != c1)) {
    for (int row = warp; row < rows; row += kFinishThreads / 32) {
      float top = -INFINITY, den = 0.0f;
      if (c0 == c1) {
        if (tiles) {
          const float2 ml = s.pair_ml[(size_t)pair * row_slots + row];
          top = ml.x;
          den = ml.y;
        }
      } else {
        for (int i = c0 + lane; i <= c1; i += 32) top = fmaxf(top, s.part_ml[(size_t)(2 * i + (i == c0)) * row_slots + row].x);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        for (int i = c0 + lane; i <= c1; i += 32) {
          const float2 ml = s.part_ml[(size_t)(2 * i + (i == c0)) * row_slots + row];
          den += ml.x == -INFINITY ? 0.0f : ml.y * exp2_fast(ml.x - top);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
      }
      if (lane == 0) {
        stat[row] = make_float2(top == -INFINITY ? 0.0f : top, top == -INFINITY ? 0.0f : 1.0f / den);
        if (blockIdx.x == 0 && c0 != c1 && s.a.lse) {
          const int i = row / s.a.group, h = head * s.a.group + row % s.a.group;
          s.a.lse[((size_t)b * s.a.tokens + i) * s.a.heads + h] = top == -INFINITY ? -INFINITY : (top + log2f(den)) * 0.6931471805599453f;
        }
      }
    }
  }
  __syncthreads();
  if (blockIdx.x == 0 && (c0 != c1 || tiles == 0)) {
    for (int x = threadIdx.x; x < rows * (D / 4); x += kFinishThreads) {
      const int row = x / (D / 4), d = x % (D / 4) * 4;
      const int i = row / s.a.group, h = head * s.a.group + row % s.a.group;
      float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (tiles) {
        const float2 st = stat[row];
#pragma unroll 8
        for (int y = c0; y <= c1; ++y) {
          const size_t at = (size_t)(2 * y + (y == c0)) * row_slots + row;
          const float m = s.part_ml[at].x;
          const float f = m == -INFINITY ? 0.0f : exp2_fast(m - st.x) * st.y;
          const float4 v = *reinterpret_cast<const float4*>(s.part_o + at * D + d);
          sum.x = fmaf(v.x, f, sum.x);
          sum.y = fmaf(v.y, f, sum.y);
          sum.z = fmaf(v.z, f, sum.z);
          sum.w = fmaf(v.w, f, sum.w);
        }
      } else if (d == 0 && s.a.lse) {
        s.a.lse[((size_t)b * s.a.tokens + i) * s.a.heads + h] = -INFINITY;
      }
      uint2 u;
      if (s.a.dtype == SPV_BF16) u = make_uint2(kv_pack2<SPV_BF16>(sum.x, sum.y), kv_pack2<SPV_BF16>(sum.z, sum.w));
      else u = make_uint2(kv_pack2<SPV_FP16>(sum.x, sum.y), kv_pack2<SPV_FP16>(sum.z, sum.w));
      *reinterpret_cast<uint2*>(s.a.o + b * s.a.o_stride_b + i * s.a.o_stride_tok + h * s.a.o_stride_head + d) = u;
    }
  }
  if (!weights) return;
  const int64_t wat = b * s.a.w_stride_b + head * s.a.w_stride_head;
#pragma unroll
  for (int x = 0; x < kFinishKeys / kFinishThreads; ++x) {
    const int key = key0 + x * kFinishThreads + threadIdx.x;
    if (key < len) {
      const float* zt = s.z + (size_t)(line + key / kTile) * s.rows * kTile + key % kTile;
      float w = 0.0f;
      if (tiles) {
#pragma unroll 8
        for (int row = 0; row < rows; ++row) w += exp2_fast(zt[row * kTile] - stat[row].x) * stat[row].y;
      }
      s.a.w_out[wat + key] = (s.a.w_in ? s.a.w_in[wat + key] : 0.0f) + w;
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------
// CTAs the plan is made for: the workspace is sized without a device, so by the largest GPU of this generation.
constexpr int kMaxCtas = 160;

int row_slots_of(int rows) { return rows <= 8 ? 8 : (rows <= 16 ? 16 : 32); }

struct Workspace { size_t part_o, part_ml, pair_ml, z, total; };
Workspace plan(const spv_kv_cache* c, const spv_kv_seqs* q, const spv_kv_attn_desc* d, bool weights) {
  const int rows = d->tokens * (d->heads / c->kv_heads), slots = row_slots_of(rows), tile = tile_of(c->head_dim);
  const size_t tiles = (size_t)q->batch * c->kv_heads * ((spv_kv_max_length(c, q) + tile - 1) / tile);
  Workspace w;
  w.part_o = 0;
  w.part_ml = w.part_o + spv_align_up((size_t)kMaxCtas * kPartSlots * slots * c->head_dim * sizeof(float), 256);
  w.pair_ml = w.part_ml + spv_align_up((size_t)kMaxCtas * kPartSlots * slots * sizeof(float2), 256);
  w.z = w.pair_ml + spv_align_up((size_t)q->batch * c->kv_heads * slots * sizeof(float2), 256);
  w.total = w.z + (weights ? spv_align_up(tiles * rows * tile * sizeof(float), 256) : 0);
  return w;
}

template <int FMT, int D, int NT>
int32_t launch(spv_ctx* ctx, int which, const CUtensorMap& mk, const CUtensorMap& mv, const KvView& view, const StreamArgs& s,
               int ctas, cudaStream_t stream) {
  constexpr int bytes = Layout<D, NT>::kTotal + 1024;
  static_assert(bytes <= 227 * 1024, "shared memory");
  static_assert(Layout<D, NT>::kOwn >= 2, "a warp works on one stage while another fills");
  auto kernel = kv_stream_kernel<FMT, D, NT>;
  if (!(ctx->kv_configured & (1u << which))) {
    SPV_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    ctx->kv_configured |= 1u << which;
  }
  kernel<<<ctas, Layout<D, NT>::kThreads, bytes, stream>>>(mk, mv, view, s);
  return cudaGetLastError() == cudaSuccess ? SPV_OK : SPV_ERR_CUDA;
}

}  // namespace

size_t spv_kv_stream_workspace(const spv_kv_cache* cache, const spv_kv_seqs* seqs, const spv_kv_attn_desc* d, bool weights) {
  return plan(cache, seqs, d, weights).total;
}

int32_t spv_kv_stream_run(spv_ctx* ctx, const spv_kv_cache* cache, const spv_kv_seqs* seqs, const KvAttnArgs& a,
                          void* workspace, cudaStream_t stream) {
  spv_kv_attn_desc d = {};
  d.tokens = a.tokens;
  d.heads = a.heads;
  const Workspace w = plan(cache, seqs, &d, a.w_out != nullptr);
  const KvView view = kv_view(ctx, cache, seqs);
  StreamArgs s;
  s.a = a;
  s.rows = a.tokens * a.group;
  char* base = (char*)workspace;
  s.part_o = (float*)(base + w.part_o);
  s.part_ml = (float2*)(base + w.part_ml);
  s.pair_ml = (float2*)(base + w.pair_ml);
  s.z = a.w_out ? (float*)(base + w.z) : nullptr;
  // a row of the map is 128 bytes: one slot of 128, or two of 64
  const uint64_t lines = (uint64_t)cache->pages * cache->kv_heads * cache->block * cache->head_dim / 128;
  const uint64_t dims[2] = {128, lines};
  const uint64_t strides[1] = {128};
  const int tile = tile_of(cache->head_dim);
  const uint32_t part = cache->block < tile ? cache->block : tile;
  const uint32_t box[2] = {128, part * cache->head_dim / 128};
  CUtensorMap mk, mv;
  int32_t st = spv_make_tmap_u8(ctx, &mk, cache->k, 2, dims, strides, box);
  if (st != SPV_OK) return st;
  if ((st = spv_make_tmap_u8(ctx, &mv, cache->v, 2, dims, strides, box)) != SPV_OK) return st;
  const int64_t most = (int64_t)seqs->batch * cache->kv_heads * ((view.max_length + tile - 1) / tile);
  int ctas = ctx->sm_count < kMaxCtas ? ctx->sm_count : kMaxCtas;
  if (most < ctas) ctas = (int)most;
  const int slots = row_slots_of(s.rows);
  auto go = [&](auto fmt, auto dim) -> int32_t {
    constexpr int base_id = (fmt() * 2 + (dim() == 128)) * 3;
    if (slots == 8) return launch<fmt(), dim(), 1>(ctx, base_id, mk, mv, view, s, ctas, stream);
    if (slots == 16) return launch<fmt(), dim(), 2>(ctx, base_id + 1, mk, mv, view, s, ctas, stream);
    return launch<fmt(), dim(), 4>(ctx, base_id + 2, mk, mv, view, s, ctas, stream);
  };
  using I8 = std::integral_constant<int, SPV_KV_INT8>;
  using E4 = std::integral_constant<int, SPV_KV_E4M3>;
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (cache->format == SPV_KV_INT8) st = cache->head_dim == 64 ? go(I8(), D64()) : go(I8(), D128());
  else st = cache->head_dim == 64 ? go(E4(), D64()) : go(E4(), D128());
  if (st != SPV_OK) return st;
  // the second kernel's launch overlaps the first; it waits on the device for the first to end
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.w_out ? (view.max_length + kFinishKeys - 1) / kFinishKeys : 1, cache->kv_heads * seqs->batch);
  cfg.blockDim = dim3(kFinishThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  SPV_CUDA_OK(cache->head_dim == 64 ? cudaLaunchKernelEx(&cfg, kv_finish_kernel<64>, view, s, ctas, slots)
                                    : cudaLaunchKernelEx(&cfg, kv_finish_kernel<128>, view, s, ctas, slots));
  return spv_launch_ok(ctx, 2);
}
