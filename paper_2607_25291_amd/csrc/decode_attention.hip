// Attention of one new token per sequence over a paged KV cache, for gfx950: split over the tokens and
// joined.
//
// A unit is (sequence, KV head, up to 16 or 32 query heads of its group). 32 keys at a time, a wave computes
// S^T = K Q^T and O^T += V^T P^T with 16x16x32 MFMAs, the query heads as columns. K operands come straight
// from the cache (lane: key l % 16, 16 bytes of its row). V operands too: lane (r, gq) reads the 16 bytes at
// columns 8 r .. 8 r + 7 of eight keys, an 8 x 8 square that 32 byte permutes turn into eight operands
// (operand e: rows d = 8 r + e, the lane's eight keys as k). Which keys those are is free as long as P has
// the same order, so they are the keys whose logits the lane holds after K Q^T: P never leaves its lanes,
// and nothing passes through LDS until a unit's end.
//
// The units' 128-token tiles form one sequence of work that a fixed grid cuts into equal ranges, whatever the lengths
// are (the host does not know them): every workgroup scans the lengths and finds its range. A
// unit that crosses ranges leaves one partial result (running maximum, sum, unnormalised O) in each, and
// a second kernel joins them in order.
//
// Bound: HBM. A token costs 512 bytes per KV head and 4 G d flops, G flops per byte. 32 / 8 heads: one sequence of 128K
// tokens (537 MB) 84 us and 4.5 us of joining, 64 of up to 64K (4.1 GB) 599 to 632 us, where a kernel that only reads
// takes 85 and 584. Values are read with loads that the caches do not keep (128K: 105 us with events, 116
// without); keys not (no gain, and 10 % slower where a short context stays in the last-level cache).
#include <float.h>

#include <algorithm>

#include "decode_device.h"
#include "decode_internal.h"
#include "decode_split.h"
#include "select_wave.h"

namespace cosa {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * 64;
constexpr int kTile = 32 * kWaves;  // tokens of a tile: 32 per wave

// A unit takes up to 16 NQ query heads of a group: NQ 1, or 2 where a group has more than 16, so that its keys and
// values are read once for all of them. Two take twice the accumulators, and one workgroup a CU instead of
// two, so they pay where every workgroup has work: 32 heads per KV head, 64 / 512 / 1024 / 2048 tiles 20.8 / 25.5 /
// 30.2 / 39.3 us (two units of 16 columns 17.1 / 24.3 / 31.3 / 42.9); 64 sequences of up to 64K, 8 KV heads 965
// (1808).
//
// 512 workgroups for 16 columns: 1024 take 96.2 us for one sequence of 128K (93.2) and 91.3 for 48 lists (83), 72.8
// for 128 sequences of up to 2K (76.3, and 63 with the slots below).
template <int NQ>
constexpr int kGrid = 512 / NQ;   // workgroups that share the tiles: as many as the CUs hold
template <int NQ>
constexpr int kRows = 16 * NQ;    // query heads of a unit
template <int NQ>
constexpr int kPartStride = kRows<NQ> * (kHeadDim + 2);  // floats of a partial result
static_assert(kGrid<1> * kPartStride<1> == kGrid<2> * kPartStride<2>, "one size of workspace");

inline int groups(int G, int nq) { return (G + 16 * nq - 1) / (16 * nq); }

struct DecodeParams {
  const uint16_t *q, *kc, *vc;
  const int32_t *table, *seq_lens, *pages, *count;
  float* part;    // [2 * grid][kPartStride<NQ>]: the partial results of a workgroup's first and last unit
  int2* rec;      // [units]: first and last workgroup of a unit that several share; first < 0: one had it all
  uint16_t* o;
  float* lse;
  int Hq, Hkv, G, QG;
  int max_pages, log2_page, list_pages;
  int items, mult;  // items of equal tile counts in a row: sequences (mult Hkv * QG) or KV heads (mult QG)
  long long q_stride, n_pages;
  float scale, scale_log2;  // of logits: natural, and for exp2
};

__device__ __forceinline__ float xmax16(float v) { return fmaxf(v, __shfl_xor(v, 16, 64)); }

__device__ __forceinline__ int seq_len(const DecodeParams& P, int n) {
  return min(max(P.seq_lens[n], 0), P.max_pages << P.log2_page);
}

// Tokens an item walks: the sequence, or its list (pages in full).
template <bool LISTED>
__device__ __forceinline__ int item_tokens(const DecodeParams& P, int i) {
  if (LISTED) return min(max(P.count[i], 0), P.list_pages) << P.log2_page;
  return seq_len(P, i);
}
__device__ __forceinline__ int tiles_of(int tokens) {
  return max((int)(((unsigned)tokens + kTile - 1) / kTile), 1);
}

// Slots of a unit in the row of work: its tiles, and what taking it up costs beside them, about one tile's time. Without
// that, ranges of many short units finish last: 128 sequences of up to 2000 tokens 82.3 us with events (71.0 with it),
// 64 of up to 4000 78.4 (72.6); one of 128K 93.6 (94.4: 17 slots for some workgroups instead of 16).
constexpr int kUnitCost = 1;
__device__ __forceinline__ int slots_of(int tokens) { return tiles_of(tokens) + kUnitCost; }

// Two fp32 weights as pairs of bf16 terms, three each, that together have all their bits. Two terms leave up to 2^-18 of a
// weight; the third one's products are free under the memory bound (two / three, events: 128K 98.0 / 97.4 to 98.2 us, 64
// sequences of up to 64K 637 / 637 to 639, with 32 heads per KV head 952 to 962 / 953 to 976).
// Every term of a weight that is not 0 is above 0, so that an infinite value gives infinity in each product and not
// NaN: the first one is the largest bf16 value below the weight (at most 17 bits are left, 16 if not a power of two), the
// second one the largest below what is left, and then 8 bits are left. (Weights below 2^-110 lose terms.)
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t (&term)[3]) {
#pragma unroll
  for (int t = 0; t < 3; ++t) {
    uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
    if (t < 2) {
      x = __builtin_elementwise_sub_sat(x, 1u) & 0xffff0000u;  // 0 stays 0
      y = __builtin_elementwise_sub_sat(y, 1u) & 0xffff0000u;
      a -= __uint_as_float(x);
      b -= __uint_as_float(y);
    }
    term[t] = __builtin_amdgcn_perm(y, x, 0x07060302u);
  }
}

// Rows of the cache as a buffer that ends behind `bytes`.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const uint16_t* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p), 0, bytes, 0x00020000);
}
constexpr int kOnce = 2;  // cache policy of a buffer load: read once, not kept

struct Tile {
  u32x4_t k[2][4], v[8];
};

// One unit's tiles [t0, t1) by the workgroup; the result goes to o and lse (part == nullptr) or to part.
template <bool LISTED, int NQ>
__device__ __forceinline__ void walk(const DecodeParams& P, int n, int g, int qg, int tokens, int t0, int t1, float* part,
                     float (*so)[kRows<NQ>][kHeadDim + 4], float (*sm)[kRows<NQ>], float (*sl)[kRows<NQ>]) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, gq = lane >> 4;
  const int rows = unit_heads(P.G, kRows<NQ>, qg);
  const int h0 = g * P.G + qg * kRows<NQ>;
  const int page = 1 << P.log2_page;
  const int len = seq_len(P, n);

  u32x4_t qf[NQ][4];
  f32x4_t acc[NQ][8];
  // Running maximum of column r and this lane's share of its sum. Maxima are kept without the scale, and differences
  // taken before it: a scaled one's rounding, 2^-24 of it, would be a factor of every weight (above 2^31, infinity or 0).
  float m[NQ], l[NQ];
#pragma unroll
  for (int x = 0; x < NQ; ++x) {
    const uint16_t* q =
        P.q + (size_t)n * P.q_stride + (size_t)(h0 + min(16 * x + r, rows - 1)) * kHeadDim + gq * 8;
#pragma unroll
    for (int c = 0; c < 4; ++c) qf[x][c] = ldg16(q + c * 32);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[x][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    m[x] = -INFINITY;
    l[x] = 0.f;
  }

  const unsigned begin = (unsigned)t0 * kTile + w * 32;
  const unsigned end = min((unsigned)t1 * kTile, (unsigned)tokens);
  const int steps = begin < end ? (int)((end - begin + kTile - 1) / kTile) : 0;
  const int32_t* row = P.table + (size_t)n * P.max_pages;
  const int32_t* list = LISTED ? P.pages + (size_t)(n * P.Hkv + g) * P.list_pages : nullptr;

  // Pages of steps i0 .. i0 + 63, one per lane: physical page and valid keys of either half (behind the last step:
  // none).
  int pg[2], valid[2];
  const auto look_up = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const unsigned pos = begin + (unsigned)(i0 + lane) * kTile + h * 16;
      pg[h] = 0;
      valid[h] = 0;
      if (i0 + lane < steps && pos < end) {
        int j = (int)(pos >> P.log2_page);
        if (LISTED) j = list[j];
        const bool in = j >= 0 && j < P.max_pages;
        const int64_t left = in ? (int64_t)len - (((int64_t)j << P.log2_page) + (pos & (unsigned)(page - 1))) : 0;
        valid[h] = (int)min(max(left, (int64_t)0), (int64_t)16);
        if (valid[h] > 0) {
          const int p = row[j];
          pg[h] = p >= 0 && p < P.n_pages ? p : 0;
        }
      }
    }
  };
  // Keys of lane-step i and of half h that count (none behind the 64 steps that were looked up).
  const auto keys_of = [&](int i, int h) __attribute__((always_inline)) {
    return __builtin_amdgcn_readlane(valid[h], i & 63) & ((i - 64) >> 31);
  };
  // The loads of a step are never branched around, so that they can stay in flight over the step before: a buffer of
  // as many rows as count gives zeros, and reads nothing, behind them.
  const auto load = [&](Tile& T, unsigned pos, int i) __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);  // one step's loads follow another's, as the waits count them
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const size_t p = (size_t)(unsigned)__builtin_amdgcn_readlane(pg[h], i & 63);
      const size_t at = (((p * P.Hkv + g) << P.log2_page) + ((pos + h * 16) & (unsigned)(page - 1))) * kHeadDim;
      const int bytes = keys_of(i, h) * (kHeadDim * 2);
      const __amdgpu_buffer_rsrc_t kr = buffer_of(P.kc + at, bytes), vr = buffer_of(P.vc + at, bytes);
#pragma unroll
      for (int c = 0; c < 4; ++c)
        T.k[h][c] = __builtin_amdgcn_raw_buffer_load_b128(kr, r * (kHeadDim * 2) + gq * 16 + c * 64, 0, 0);
#pragma unroll
      for (int c = 0; c < 4; ++c)
        T.v[h * 4 + c] =
            __builtin_amdgcn_raw_buffer_load_b128(vr, gq * 4 * (kHeadDim * 2) + r * 16 + c * (kHeadDim * 2), 0, kOnce);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  const auto compute = [&](Tile& T, int v0, int v1) __attribute__((always_inline)) {
    u32x4_t pt[NQ][3];  // the weights' bf16 terms
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      f32x4_t s[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < 4; ++c) s[h] = mfma16(T.k[h][c], qf[x][c], s[h]);
      }
      if (v0 < 16 || v1 < 16) {  // keys behind the sequence (read as zeros, as their values are): no weight
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (gq * 4 + i >= (h ? v1 : v0)) s[h][i] = -INFINITY;
      }
      float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                       fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
      mx = half_max(xmax16(mx));
      const float mn = fmaxf(m[x], mx);
      const float base = mn == -INFINITY ? 0.f : mn;
      const float alpha = __builtin_amdgcn_exp2f((m[x] - base) * P.scale_log2);
      float p[8], sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f((s[i >> 2][i & 3] - base) * P.scale_log2);
        sum += p[i];
      }
      l[x] = l[x] * alpha + sum;
      m[x] = mn;
      if (__any(alpha != 1.f)) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[x][e][i] *= alpha;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t term[3];
        split_bf16(p[2 * i], p[2 * i + 1], term);
#pragma unroll
        for (int t = 0; t < 3; ++t) pt[x][t][i] = term[t];
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // operand e: element e of the lane's eight keys
      u32x4_t a;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        a[i] = __builtin_amdgcn_perm(T.v[2 * i + 1][e >> 1], T.v[2 * i][e >> 1],
                                     (e & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int x = 0; x < NQ; ++x)
#pragma unroll
        for (int t = 0; t < 3; ++t) acc[x][e] = mfma16(a, pt[x][t], acc[x][e]);
    }
  };

  for (int i0 = 0; i0 < steps; i0 += 64) {
    const int n_steps = min(steps - i0, 64);
    const unsigned pos = begin + (unsigned)i0 * kTile;
    Tile A, B;
    look_up(i0);
    load(A, pos, 0);
    load(B, pos + kTile, 1);
    int i = 0;
    for (; i + 1 < n_steps; i += 2) {
      compute(A, keys_of(i, 0), keys_of(i, 1));
      load(A, pos + (unsigned)(i + 2) * kTile, i + 2);
      compute(B, keys_of(i + 1, 0), keys_of(i + 1, 1));
      load(B, pos + (unsigned)(i + 3) * kTile, i + 3);
    }
    if (i < n_steps) compute(A, keys_of(i, 0), keys_of(i, 1));
  }

  // The waves' results: lane (r, gq) holds columns d = 8 (4 gq + i) + e of query head r.
#pragma unroll
  for (int x = 0; x < NQ; ++x) {
    float sum = l[x] + __shfl_xor(l[x], 16, 64);
    sum = half_sum(sum);
    const int row = 16 * x + r;
    if (row < rows) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float* to = &so[w][row][8 * (4 * gq + i)];
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e] = acc[x][e][i];
      }
      if (gq == 0) {
        sm[w][row] = m[x];
        sl[w][row] = sum;
      }
    }
  }
  __syncthreads();
  for (int x = threadIdx.x; x < rows * kHeadDim; x += kThreads) {
    const int hh = x >> 7, d = x & 127;
    float M = sm[0][hh];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) M = fmaxf(M, sm[i][hh]);
    const float base = M == -INFINITY ? 0.f : M;
    float L = 0.f, O = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const float a = __builtin_amdgcn_exp2f((sm[i][hh] - base) * P.scale_log2);
      L += a * sl[i][hh];
      O += a * so[i][hh][d];
    }
    if (part) {
      part[hh * kHeadDim + d] = O;
      if (d == 0) {
        part[kRows<NQ> * kHeadDim + hh] = M;
        part[kRows<NQ> * (kHeadDim + 1) + hh] = L;
      }
    } else {
      const size_t out = (size_t)n * P.Hq + h0 + hh;
      // nothing to attend to: 0 (a sum that is NaN, from a NaN logit, stays NaN)
      const __bf16 v = (__bf16)(L == 0.f ? 0.f : O / L);
      P.o[out * kHeadDim + d] = __builtin_bit_cast(uint16_t, v);
      if (P.lse && d == 0) P.lse[out] = L == 0.f ? -INFINITY : M * P.scale + logf(L);
    }
  }
  __syncthreads();  // so, sm and sl are used again
}

// Tiles [begin, end) of workgroup w of n, of `all` tiles: the first all % n workgroups have one more than the others.
struct Range {
  uint32_t begin, end;
};
__device__ __forceinline__ Range range_of(uint32_t w, uint32_t n, uint32_t all) {
  const uint32_t q = all / n, r = all % n;
  const uint32_t begin = w * q + min(w, r);
  return {begin, begin + q + (w < r)};
}
// The workgroup whose range holds tile x.
__device__ __forceinline__ int owner_of(uint32_t x, uint32_t n, uint32_t all) {
  const uint32_t q = all / n, r = all % n, big = r * (q + 1);
  return (int)(x < big ? x / (q + 1) : r + (x - big) / q);
}

// WHOLE: a workgroup per unit, no splitting.
template <bool LISTED, bool WHOLE, int NQ>
__global__ __launch_bounds__(kThreads, 2 / NQ) void decode_kernel(DecodeParams P) {
  __shared__ float so[kWaves][kRows<NQ>][kHeadDim + 4], sm[kWaves][kRows<NQ>], sl[kWaves][kRows<NQ>];
  const auto unit = [&](int item, int sub, int t0, int t1, int tokens, float* part) __attribute__((always_inline)) {
    const int n = LISTED ? item / P.Hkv : item;
    const int g = LISTED ? item % P.Hkv : sub / P.QG;
    walk<LISTED, NQ>(P, n, g, sub % P.QG, tokens, t0, t1, part, so, sm, sl);
  };
  if (WHOLE) {
    const int item = blockIdx.x / P.mult;
    const int tokens = item_tokens<LISTED>(P, item);
    unit(item, blockIdx.x % P.mult, 0, tiles_of(tokens), tokens, nullptr);
    return;
  }
  // Tiles of the items before each lane's share of them, and all tiles.
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint32_t total, before;  // all tiles; tiles in front of the item
  int item;
  Range R;
  if (P.items <= 64) {  // one item a lane: every wave for itself
    const uint32_t t = lane < P.items ? (uint32_t)slots_of(item_tokens<LISTED>(P, lane)) : 0u;
    const uint32_t at = wave_incl_scan(t, lane) - t;
    total = __builtin_amdgcn_readlane(at + t, 63);
    R = range_of(blockIdx.x, gridDim.x, total * P.mult);
    item = __builtin_popcountll(__ballot(lane < P.items && at <= R.begin / (uint32_t)P.mult)) - 1;
    before = __builtin_amdgcn_readlane(at, item);
  } else {
    __shared__ uint32_t waves[kWaves];
    __shared__ int found[2];
    const int per = (P.items + kThreads - 1) / kThreads;
    const int i0 = min((int)threadIdx.x * per, P.items), i1 = min(i0 + per, P.items);
    uint32_t sum = 0;
    for (int i = i0; i < i1; ++i) sum += (uint32_t)slots_of(item_tokens<LISTED>(P, i));
    const uint32_t incl = wave_incl_scan(sum, lane);
    if (lane == 63) waves[w] = incl;
    __syncthreads();
    uint32_t at = incl - sum;
    total = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      if (i < w) at += waves[i];
      total += waves[i];
    }
    R = range_of(blockIdx.x, gridDim.x, total * P.mult);
    const uint32_t x = R.begin / (uint32_t)P.mult;
    if (x >= at && x < at + sum) {
      int i = i0;
      for (;; ++i) {
        const uint32_t t = (uint32_t)slots_of(item_tokens<LISTED>(P, i));
        if (x < at + t) break;
        at += t;
      }
      found[0] = i;
      found[1] = (int)at;
    }
    __syncthreads();
    item = __builtin_amdgcn_readfirstlane(found[0]);
    before = __builtin_amdgcn_readfirstlane(found[1]);
  }
  uint32_t a = R.begin;
  const uint32_t b = R.end;
  if (a == b) return;
  int tokens = item_tokens<LISTED>(P, item);
  int tiles = tiles_of(tokens);
  const uint32_t rem = a - before * P.mult, slots = (uint32_t)tiles + kUnitCost;
  int sub = (int)(rem / slots), t0 = (int)(rem % slots);
  for (;;) {
    if (t0 < tiles) {
      const int t1 = (int)min((uint32_t)t0 + (b - a), (uint32_t)tiles);
      float* part = nullptr;
      if (t0 > 0 || t1 < tiles) part = P.part + ((size_t)blockIdx.x * 2 + (t0 == 0)) * kPartStride<NQ>;
      if (t0 == 0 && threadIdx.x == 0)
        P.rec[item * P.mult + sub] =
            t1 < tiles ? int2{(int)blockIdx.x, owner_of(a + tiles - 1, gridDim.x, total * P.mult)} : int2{-1, 0};
      unit(item, sub, t0, t1, tokens, part);
    }
    if (b - a <= (uint32_t)(tiles + kUnitCost - t0)) return;
    a += tiles + kUnitCost - t0;
    t0 = 0;
    if (++sub == P.mult) {
      sub = 0;
      tokens = item_tokens<LISTED>(P, ++item);
      tiles = tiles_of(tokens);
    }
  }
}

constexpr int kJoinThreads = 32 * kJoinGroups;

// Joins the partial results of unit blockIdx.x, for `heads` query heads from blockIdx.y * heads on. A group of 32
// threads adds partial results, four columns a thread; the 16 groups are dealt to the heads and, within a
// head, to its partial results in turn, so that the loads of many wait side by side.
template <bool LISTED, int NQ>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(DecodeParams P, int heads, int log2_per_head) {
  __shared__ f32x4_t sums[kJoinGroups][32];
  __shared__ float lsum[kJoinGroups], tops[kJoinGroups];
  const int2 rec = P.rec[blockIdx.x];
  if (rec.x < 0) return;
  const int item = blockIdx.x / P.mult, sub = blockIdx.x % P.mult;
  const int n = LISTED ? item / P.Hkv : item, g = LISTED ? item % P.Hkv : sub / P.QG, qg = sub % P.QG;
  const int t = threadIdx.x & 31, group = threadIdx.x >> 5;
  const int per_head = 1 << log2_per_head, mine = group & (per_head - 1);
  const int hh = join_head(heads, log2_per_head, unit_heads(P.G, kRows<NQ>, qg), blockIdx.y, group);
  const bool live = hh >= 0;
  const int first = rec.x, n_parts = rec.y - first + 1;
  const auto part = [&](int i) { return P.part + ((size_t)(first + i) * 2 + (i == 0)) * kPartStride<NQ>; };
  float M = -INFINITY, L = 0.f;
  f32x4_t O = {0.f, 0.f, 0.f, 0.f};
  const auto add = [&](float m, float l, const f32x4_t& o) {
    const float mx = fmaxf(M, m), base = mx == -INFINITY ? 0.f : mx;
    const float a = __builtin_amdgcn_exp2f((M - base) * P.scale_log2), b = __builtin_amdgcn_exp2f((m - base) * P.scale_log2);
    L = a * L + b * l;
    O = a * O + b * o;
    M = mx;
  };
  if (live) {
    for (int i0 = mine; i0 < n_parts; i0 += 4 * per_head) {
      float m[4], l[4];
      f32x4_t o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // behind the last part: that one again, without weight
        const float* p = part(min(i0 + i * per_head, n_parts - 1));
        m[i] = p[kRows<NQ> * kHeadDim + hh];
        l[i] = p[kRows<NQ> * (kHeadDim + 1) + hh];
        o[i] = *reinterpret_cast<const f32x4_t*>(p + hh * kHeadDim + t * 4);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i0 + i * per_head < n_parts) add(m[i], l[i], o[i]);
    }
    sums[group][t] = O;
    if (t == 0) {
      lsum[group] = L;
      tops[group] = M;
    }
  }
  __syncthreads();
  if (!live || mine != 0) return;
  for (int i = 1; i < per_head; ++i) add(tops[group + i], lsum[group + i], sums[group + i][t]);
  const size_t out = (size_t)n * P.Hq + (size_t)g * P.G + qg * kRows<NQ> + hh;
  uint16_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = __builtin_bit_cast(uint16_t, (__bf16)(L == 0.f ? 0.f : O[i] / L));
  *reinterpret_cast<u32x2_t*>(P.o + out * kHeadDim + t * 4) =
      u32x2_t{o[0] | (uint32_t)o[1] << 16, o[2] | (uint32_t)o[3] << 16};
  if (P.lse && t == 0) P.lse[out] = L == 0.f ? -INFINITY : M * P.scale + logf(L);
}

template <bool LISTED, int NQ>
hipError_t launch_t(const DecodeParams& P, long long tokens, hipStream_t stream) {
  const long long units = (long long)P.items * P.mult, tiles = (tokens + kTile - 1) / kTile;
  // A workgroup for every unit, and no join, where a unit is short, or less short and there are enough of them: 8
  // units of 256 / 512 / 1000 tokens 11.7 / 13.8 / 18.0 us (split 16.2 / 16.3 / 16.3); 256 units of 512 / 1000
  // 19.3 / 28.2 (24.6 / 32.5), 320 of them 25.0 / 38.5 (28.0 / 39.6), 800 of them 42.4 / 80.8 (46.6 / 82.7); of 2000
  // tokens 46.4 / 71.3 / 150 (50.0 / 67.0 / 148).
  if (tokens <= 512 || (tokens <= 1024 && units >= 256)) {
    hipLaunchKernelGGL((decode_kernel<LISTED, true, NQ>), dim3((unsigned)units), dim3(kThreads), 0, stream, P);
    return hipGetLastError();
  }
  const int grid = (int)std::min<long long>(units * tiles, kGrid<NQ>);
  hipLaunchKernelGGL((decode_kernel<LISTED, false, NQ>), dim3(grid), dim3(kThreads), 0, stream, P);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const JoinShape j = join_shape(units, P.G, kRows<NQ>);
  hipLaunchKernelGGL((join_kernel<LISTED, NQ>), dim3((unsigned)units, j.groups), dim3(kJoinThreads), 0, stream, P, j.heads,
                     j.log2_per_head);
  return hipGetLastError();
}

}  // namespace

// The workspace: a record per unit, then two partial results per workgroup.
static size_t record_bytes(const DecodeShape& sh) {
  return ((size_t)sh.B * sh.Hkv * groups(sh.G, 1) * sizeof(int2) + 255) / 256 * 256;
}

size_t decode_workspace_bytes(const DecodeShape& sh) {
  return record_bytes(sh) + (size_t)kGrid<1> * 2 * kPartStride<1> * sizeof(float);
}

bool decode_fits(const DecodeShape& sh, long long tokens) {
  const long long units = (long long)sh.B * sh.Hkv * groups(sh.G, 1), tiles = std::max<long long>((tokens + kTile - 1) / kTile, 1) + kUnitCost;
  // 2^32 threads of a grid, in workgroups of up to 1024; tiles in 31 bits
  return units < (1ll << 22) && units * tiles < (1ll << 31);
}

hipError_t launch_decode_attention(const DecodeShape& sh, const DecodeArgs& a, hipStream_t stream) {
  const bool listed = a.pages != nullptr;
  // Selected lists are wider than 2^31 tokens only by entries that their counts never reach.
  const long long tokens = listed ? std::min((long long)a.list_pages << sh.log2_page, 0x7fffffffll) : sh.cap();
  const int nq = sh.G > 16 && (long long)sh.B * sh.Hkv * ((tokens + kTile - 1) / kTile) > kGrid<1> ? 2 : 1;
  const int QG = groups(sh.G, nq);
  int2* rec = static_cast<int2*>(a.workspace);
  float* part = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + record_bytes(sh));
  const DecodeParams P{a.q, a.k_cache, a.v_cache, a.table, a.seq_lens, a.pages, a.count, part, rec, a.o, a.lse,
                       sh.Hq, sh.Hkv, sh.G, QG, sh.max_pages, sh.log2_page, a.list_pages,
                       listed ? sh.B * sh.Hkv : sh.B, listed ? QG : sh.Hkv * QG, sh.q_stride, sh.n_pages,
                       sh.scale, std::min(sh.scale * 1.4426950408889634f, FLT_MAX)};  // 0 times infinity is no logit
  if (nq == 1) return listed ? launch_t<true, 1>(P, tokens, stream) : launch_t<false, 1>(P, tokens, stream);
  return listed ? launch_t<true, 2>(P, tokens, stream) : launch_t<false, 2>(P, tokens, stream);
}

}  // namespace cosa
