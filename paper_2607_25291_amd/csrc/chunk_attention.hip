// Attention of chunks of new tokens over a paged KV cache, for gfx950: causal from each sequence's end, split
// over the keys and joined.
//
// A unit (chunk_split.h) has 256 rows, whole tokens of all query heads of a KV head, so that keys and values are fetched
// once for the group. Eight waves of 32 rows each walk the keys in tiles of 128: S^T = K Q^T with 32x32x16 MFMAs, so that a
// lane owns a row, an online softmax in fp32 and O^T += V^T P^T, whose P^T operand the lane holds already. Tiles go
// from the pages straight into LDS (buffer loads with an LDS destination), double-buffered; a wave moves runs of 16
// rows, which lie in one page whatever its size, through buffers that end behind the last key, so that rows behind it are
// zeros.
//
// The units' slots form one line that a fixed grid cuts into equal ranges on the device (the host knows no
// lengths); a unit in several ranges leaves partial results (running maximum, sum, unnormalised O), which a second
// kernel joins in order.
//
// o = sum_t exp(s_t - M) v_t / sum_t exp(s_t - M), in one pass: where a larger maximum comes, what is summed so far is
// multiplied by exp(old - new). Weights are rounded to bf16 for the product with V, as in the prefill (at most half a step, 2^-8,
// of a weight; their sum takes them with 24 bits): the further bits would be products of their own, and MFMA is what bounds large
// units. Units of few rows, which memory bounds, round alike: a token's weights do not depend on what shares its unit. The
// results' error against 64 bits grows by 0.5 to 2 % over that of their last rounding to bf16 (1.65e-3 to 1.68e-3, 19 prompts).
//
// Bound: MFMA, 4 d flops a key and row. 4096 tokens over 64K, 32 / 8 heads: 3.7 to 3.9 ms, 1.13 PFLOP/s where a library matrix
// product of 8192 rows takes 1.24; 0.59 of the cycles multiply at 1.78 GHz, LDS bank conflicts are below 0.1 %. 256 rows: eight
// waves share a tile's copies, and two waves a SIMD, one phase apart, let one multiply while the other one takes
// exponentials. What a unit costs beside its tiles (3 tiles: edges, results, a side that waits for the other one's) leaves
// 840 to 880 TFLOP/s in prompts of up to 4K tokens. Units of few rows wait for the 64 KiB of one tile at a time: 5.6 TB/s (64
// sequences of up to 64K tokens and one new token 292 us). The smallest calls (16 new ones of 1000 tokens, 4 heads, 16 us) are
// two launches and latency.
#include <float.h>
#include <limits.h>
#include <math.h>
#include <stddef.h>

#include <algorithm>
#include <type_traits>

#include "chunk_split.h"
#include "cosa_device.h"
#include "serving_internal.h"

namespace cosa {
namespace {

constexpr int kWaves = 8, kThreads = kWaves * 64;
constexpr int kTile = kChunkTile;
constexpr int kKeyTiles = kTile / 32;
constexpr int kTileBytes = kTile * kHeadDim * 2;  // one tensor's
constexpr int kLog2Grid = 8, kGrid = 1 << kLog2Grid;  // workgroups that share the line: one a CU
// Slots of the shortest range: at least a tile's. Shorter ones end sooner and leave more to join: 384 / 512 slots 18.1 / 19.4 us
// for 8 rows over 4K tokens, 16.4 / 16.1 for 16 over 1000 and 26.2 / 24.0 for 2 rows of 20 heads over 49K; 0.5 % for 512 over 8K.
constexpr int kShortest = 512;
static_assert(kShortest >= kTile * kFullSlots, "every range but the last holds the start of a tile");
constexpr int kRowFloats = kHeadDim + 2;          // of a partial result: O, maximum, sum

// Partial results of workgroup b: slot 2 b of its first unit, which began in a range before, 2 b + 1 of its last one.
struct ChunkParams {
  const uint16_t *q, *kc, *vc;
  const int32_t *table, *seq_lens, *cu_new;
  float* part;
  // [kGrid]: a unit that begins in range b and ends in another one: first row, rows, head and part, last range; or, where range
  // b lies inside a unit: the range in which that begins, -1; or 0, 0
  int4* rec;
  uint16_t* o;
  float* lse;
  int B, Hq, Hkv, G, GP, parts, T;  // GP: heads of a unit
  int max_pages, log2_page, n_rows, part_rows, log2_grid;
  long long q_stride, n_pages;
  float scale, scale_log2;
};

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// Sequence n as its units see it, and its first row.
__device__ __forceinline__ ChunkSeq seq_of(const ChunkParams& P, int cu0, int cu1, int len, int& row0) {
  row0 = min(max(cu0, 0), P.n_rows);
  const int end = min(max(cu1, row0), P.n_rows);
  return {min(max(len, 0), P.max_pages << P.log2_page), end - row0, P.T, P.GP};
}
__device__ __forceinline__ ChunkSeq seq_of(const ChunkParams& P, int n) {
  int row0;
  return seq_of(P, P.cu_new[n], P.cu_new[n + 1], P.seq_lens[n], row0);
}

// Uniform reads of data that the kernels never write, through the constant address space: scalar loads.
__device__ __forceinline__ int32_t ld_uniform(const int32_t* p) {
  return *(const __attribute__((address_space(4))) int32_t*)(size_t)p;
}
// Values that are the same in every lane, in scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)x) | (int64_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32;
}

__device__ __forceinline__ ChunkSeq seq_of_uniform(const ChunkParams& P, int n, int& row0) {
  const ChunkSeq S = seq_of(P, ld_uniform(P.cu_new + n), ld_uniform(P.cu_new + n + 1), ld_uniform(P.seq_lens + n), row0);
  row0 = uniform(row0);
  return {uniform(S.len), uniform(S.w), P.T, P.GP};
}

// The first sequence from n on that has rows; P.B if none has. 256 at a time, four a lane: one by one, a batch of 512 / 8192 slots
// of which the first and the last are busy takes 68 / 868 us, now 17 / 28 (16.6 / 19.7 where they lie side by side).
__device__ __forceinline__ int next_with_rows(const ChunkParams& P, int n) {
  const int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  for (; n < P.B; n += 4 * 64) {
    int32_t from[4], to[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = min(n + 64 * k + lane, P.B - 1);  // behind the last one: that one again, which its own lane finds first
      from[k] = P.cu_new[i];
      to[k] = P.cu_new[i + 1];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint64_t busy = __ballot(min(to[k], P.n_rows) > max(from[k], 0));
      if (busy) return uniform(n + 64 * k + (int)__builtin_ctzll(busy));
    }
  }
  return P.B;
}

// Heads of unit part hp of a group.
__device__ __forceinline__ int heads_of(const ChunkParams& P, int hp) { return min(P.G - hp * P.GP, P.GP); }

// A value that is formed again where it is used, not held in a register over the walk.
__device__ __forceinline__ int again(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Four results as bf16.
__device__ __forceinline__ void store4(uint16_t* to, const float (&x)[4]) {
  uint32_t w[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const __bf16 lo = (__bf16)x[2 * e], hi = (__bf16)x[2 * e + 1];
    w[e] = (uint32_t)__builtin_bit_cast(uint16_t, lo) | ((uint32_t)__builtin_bit_cast(uint16_t, hi) << 16);
  }
  *reinterpret_cast<u32x2_t*>(to) = u32x2_t{w[0], w[1]};
}

// The rounded m c that weights refer to, and what takes sums of such weights to the exact one.
__device__ __forceinline__ float rounded(float m, float c) {
#pragma clang fp contract(off)
  return m * c;
}
__device__ __forceinline__ float exact_by(float m, float c) { return __builtin_amdgcn_exp2f(-fmaf(m, c, -rounded(m, c))); }
constexpr float kLn2 = 0.69314718f;
constexpr float kFar = 65536.f;  // the factor is within 2^-8 of 1 below

// End of a phase: LDS accesses done (and, with full, this wave's copies landed), then the workgroup barrier.
__device__ __forceinline__ void end_phase(bool full) {
  if (full) __builtin_amdgcn_s_waitcnt(kVmcntLgkm0);
  else __builtin_amdgcn_s_waitcnt(kLgkm0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

struct Lds {
  char v[2][kTileBytes];  // the low 64 KiB: every transposing read's offsets fit its immediate
  char k[2][kTileBytes];
  int32_t unit[4][4][16];  // units in turn, a copy for the two waves of a SIMD: side 0 writes them
  int32_t pages[4][2][64]; // of the next unit's first tiles: a wave's two runs, a tile each
  int64_t range[3];             // the range's first slot and its end, and the length of all ranges
  int row[kChunkRows];  // token and head of a row, for units of GP heads: token << 16 | head
  alignas(16) int odd[2][4];  // whether a wave's part of the V tile holds an infinite or NaN value (tiles that not all rows see)
};
static_assert(offsetof(Lds, v) % 1024 == 0 && offsetof(Lds, k) % 1024 == 0 && offsetof(Lds, unit) % 16 == 0 &&
                  offsetof(Lds, range) % 8 == 0 && offsetof(Lds, odd) % 16 == 0,
              "what is read and written 16 bytes at a time lies at multiples of 16 bytes");

// A unit of the line and the range's tiles of it. I: the type of slots, 32 bits where they hold all of them (8 rows over 4K
// tokens 19 us, with 64 bits 0.4 more).
template <class I>
struct Unit {
  ChunkSeq S;
  int n, row0;  // sequence, its first row
  int g, hp, j; // KV head, part of its group, unit of these
  I at;         // its first slot
  int tiles, t0, t1;
};
// Units wait in LDS: in scalar registers, two of them would push other values out.
template <class I>
__device__ __forceinline__ void put(int32_t* to, const Unit<I>& u) {
  if ((threadIdx.x & 63) == 0) {
    int4* p = reinterpret_cast<int4*>(to);
    p[0] = int4{u.S.len, u.S.w, u.n, u.row0};
    p[1] = int4{u.g, u.j, (int)u.at, (int)((int64_t)u.at >> 32)};
    p[2] = int4{u.tiles, u.t0, u.t1, u.hp};
  }
}
template <class I>
__device__ __forceinline__ Unit<I> get(const int32_t* from, const ChunkParams& P) {
  asm volatile("" ::: "memory");
  const int4* p = reinterpret_cast<const int4*>(from);
  const int4 a = p[0], b = p[1], c = p[2];
  return {{uniform(a.x), uniform(a.y), P.T, P.GP}, uniform(a.z), uniform(a.w), uniform(b.x), uniform(c.w), uniform(b.y),
          uniform((I)((int64_t)(uint32_t)b.z | (int64_t)b.w << 32)), uniform(c.x), uniform(c.y), uniform(c.z)};
}

template <class I>
__global__ __attribute__((amdgpu_flat_work_group_size(kThreads, kThreads))) __attribute__((amdgpu_waves_per_eu(2, 2)))
void chunk_kernel(const ChunkParams P) {
  __shared__ __attribute__((aligned(1024))) Lds lds;
  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
  const int w = uniform((int)threadIdx.x >> 6);

  // The range of this workgroup, and its first unit. Slots of the sequences: one a lane, every wave for itself, or a
  // stretch of them a thread.
  const int all_heads = P.Hkv * P.parts;
  int cu0 = 0, cu1 = 0, tokens = 0;
  if (P.B <= 64 && lane < P.B) {
    cu0 = P.cu_new[lane];
    cu1 = P.cu_new[lane + 1];
    tokens = P.seq_lens[lane];
  }
  {  // while these load
    const int x = w * 32 + l32, tok = x / P.GP;
    lds.row[x] = tok << 16 | (x - tok * P.GP);
  }
  Unit<I> D;
  I begin, end, total = 0;
  int b;
  const auto place = [&]() __attribute__((always_inline)) {
    const I length = chunk_range<I>(total, P.log2_grid, kShortest);
    // Neighbouring ranges, which mostly share a KV head, go to one XCD: of all ranges, or of those with slots.
    const int per_xcd = length > kShortest ? gridDim.x / kNumXcd : (int)((total + kShortest * kNumXcd - 1) / (kShortest * kNumXcd));
    const int k = blockIdx.x / kNumXcd;
    b = k < per_xcd ? (blockIdx.x % kNumXcd) * per_xcd + k : (int)blockIdx.x;
    begin = k < per_xcd ? min((I)b * length, total) : total;
    end = min(begin + length, total);
    if (threadIdx.x == 0) {
      P.rec[b] = int4{0, 0, 0, 0};
      lds.range[0] = begin;
      lds.range[1] = end;
      lds.range[2] = length;
    }
  };
  const auto of = [&](I x, int l) __attribute__((always_inline)) -> I {
    if (sizeof(I) == 4) return __builtin_amdgcn_readlane((int)x, l);
    return (I)((int64_t)(uint32_t)__builtin_amdgcn_readlane((int)x, l) |
               (int64_t)__builtin_amdgcn_readlane((int)((int64_t)x >> 32), l) << 32);
  };
  const auto scan = [&](I x) __attribute__((always_inline)) -> I {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const I y = (I)__shfl_up(x, d, 64);
      if (lane >= d) x += y;
    }
    return x;
  };
  if (P.B <= 64) {
    int row0;
    ChunkSeq S = seq_of(P, cu0, cu1, tokens, row0);
    if (lane >= P.B) S.w = 0;
    const I mine = S.template slots<I>() * all_heads;
    const I at = P.B == 1 ? mine : scan(mine);
    total = of(at, P.B - 1);
    place();
    if (begin >= total) return;
    D.n = __builtin_popcountll(__ballot(lane < P.B && at <= begin));  // the sequences that end in front of it
    D.at = of(at - mine, D.n);
    D.S = ChunkSeq{__builtin_amdgcn_readlane(S.len, D.n), __builtin_amdgcn_readlane(S.w, D.n), P.T, P.GP};
    D.row0 = __builtin_amdgcn_readlane(row0, D.n);
  } else {
    __shared__ I sums[kWaves];
    __shared__ I found_at;
    __shared__ int found;
    const int per = (P.B + kThreads - 1) / kThreads;
    const int n0 = min((int)threadIdx.x * per, P.B), n1 = min(n0 + per, P.B);
    I mine = 0;
    for (int n = n0; n < n1; ++n) mine += seq_of(P, n).template slots<I>() * all_heads;
    I at = scan(mine);
    if (lane == 63) sums[w] = at;
    __syncthreads();
    at -= mine;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      if (i < w) at += sums[i];
      total += sums[i];
    }
    total = uniform(total);
    place();
    if (begin >= total) return;
    if (begin >= at && begin < at + mine) {
      int n = n0;
      for (; n < n1 - 1; ++n) {
        const I t = seq_of(P, n).template slots<I>() * all_heads;
        if (begin < at + t) break;
        at += t;
      }
      found = n;
      found_at = at;
    }
    __syncthreads();
    D.n = uniform(found);
    D.at = uniform(found_at);
    D.S = seq_of_uniform(P, D.n, D.row0);
  }
  {
    // largest i in [0, n) with start(i) <= x
    const auto search = [&](int n, I x, auto&& start) __attribute__((always_inline)) -> int {
      int first = 0;
      for (int step = search_step(n); step; step /= 64) {
        const int64_t i = (int64_t)first + (int64_t)lane * step;
        first += (__builtin_popcountll(__ballot(i < n && start((int)i) <= x)) - 1) * step;
      }
      return first;
    };
    const I one = uniform(D.S.template slots<I>());
    const int hh = all_heads == 1 ? 0 : uniform(search(all_heads, begin - D.at, [&](int i) { return one * i; }));
    D.g = P.parts == 1 ? hh : uniform(hh / P.parts);
    D.hp = hh - D.g * P.parts;
    D.at += hh * one;
    const int units = uniform(D.S.units());
    D.j = units == 1 ? 0 : uniform(search(units, begin - D.at, [&](int i) { return D.S.template start<I>(i); }));
    D.at = uniform(D.at + D.S.template start<I>(D.j));
  }
  const auto settle = [&](Unit<I>& u, I begin, I end) __attribute__((always_inline)) {
    u.tiles = uniform(u.S.tiles(u.j));
    const int key_slots = u.S.key_slots(u.j);
    u.t0 = uniform(chunk_tile0<I>(begin, u.at, key_slots));
    u.t1 = uniform(chunk_tile1<I>(end, u.at, key_slots, u.tiles));
  };
  // The next unit of the range (its first one may have no tile here).
  const auto advance = [&](Unit<I>& u, I begin, I end) __attribute__((always_inline)) -> bool {
    u.at = uniform(u.at + u.S.template cost<I>(u.j));
    if (u.at >= end) return false;
    if (++u.j == u.S.units()) {
      u.j = 0;
      if (++u.hp == P.parts) {
        u.hp = 0;
        ++u.g;
      }
      if (u.g == P.Hkv) {
        u.g = 0;
        if (++u.n >= P.B) return false;
        u.S = seq_of_uniform(P, u.n, u.row0);
        if (u.S.w == 0) {  // there are slots left, so there is another sequence with rows
          u.n = next_with_rows(P, u.n + 1);
          if (u.n >= P.B) return false;
          u.S = seq_of_uniform(P, u.n, u.row0);
        }
      }
    }
    settle(u, begin, end);
    return true;
  };
  settle(D, begin, end);
  if (D.t0 >= D.t1 && !advance(D, begin, end)) return;

  // Copies. Waves w and w + 4 share a SIMD; side 1 (w >= 4) runs one phase behind. Side 0 moves K, side 1 V: wave wl rows 32
  // wl .. 32 wl + 31 of a tile, in two runs of 16. A lane fills slot lane % 16 of row lane / 16 of four rows with the
  // slot that the layout puts there (K: slot ^ row % 16, V: slot ^ 4 (row % 4), as the MFMA operand and the transposing
  // reads want them).
  const int side = w >> 2, wl = w & 3;
  const uint64_t head_bytes = (uint64_t)(kHeadDim * 2) << P.log2_page;
  const uint64_t page_bytes = head_bytes * (uint64_t)P.Hkv;
  const int page_mask = (1 << P.log2_page) - 1;
  const int lane_off = (lane >> 4) * 256 + (((lane & 15) ^ (side ? (lane >> 4) << 2 : lane >> 4)) << 4);
  const int step_off = side ? 0 : 64;  // K: slots of rows 4 further on differ in two more bits
  // The unit whose tiles are fetched: its keys, its KV head's cache, and its first token's place.
  int f_keys, f_first;
  uint64_t f_cache;
  const int32_t* f_row;
  int pg[2];
  const auto fetch_from = [&](const Unit<I>& u) __attribute__((always_inline)) {
    f_keys = uniform(u.S.keys(u.j));
    f_first = u.S.len - u.S.w + u.j * P.T;
    f_cache = (uint64_t)uniform((int64_t)((uint64_t)(side ? P.vc : P.kc) + (uint64_t)u.g * head_bytes));
    f_row = P.table + (size_t)u.n * P.max_pages;
  };
  // Physical pages of the runs of tiles t .. t + 63, one tile a lane (run r: rows 32 wl + 16 r).
  // Behind the last key the last entry is read again (no branch in which lanes part: what follows stays uniform).
  const auto page_of = [&](const int32_t* row, int keys, int t, int r) __attribute__((always_inline)) -> int {
    if (keys <= 0) return 0;
    const int64_t x = (int64_t)(t + again(lane)) * kTile + wl * 32 + r * 16;
    return row[min(x, (int64_t)keys - 1) >> P.log2_page];
  };
  const auto look_up = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 2; ++r) pg[r] = page_of(f_row, f_keys, t, r);
  };
  const auto copy = [&](int t, int i, int buf) __attribute__((always_inline)) {
    char* dst = (side ? lds.v[0] : lds.k[0]) + buf * kTileBytes + wl * 32 * 256;
    const int off = again(lane_off);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int x = t * kTile + wl * 32 + r * 16;  // below 2^31 + 128 where it holds a key
      const int valid = uniform(min(max(f_keys - x, 0), 16));
      const uint32_t e = (uint32_t)__builtin_amdgcn_readlane(pg[r], i & 63);
      const uint64_t p = e < (uint64_t)P.n_pages ? e : 0u;
      const uint64_t base = f_cache + p * page_bytes + (uint64_t)(x & page_mask) * (kHeadDim * 2);
      const __amdgpu_buffer_rsrc_t rs =
          __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, valid * (kHeadDim * 2), 0x00020000);
      const auto to = COSA_LDS(dst + r * 16 * 256);
      // the immediate offset counts for the bounds and moves both addresses
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, to, 16, off, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, to, 16, off ^ step_off, 0, 1024, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, to, 16, off ^ (2 * step_off), 0, 2 * 1024, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, to, 16, off ^ (3 * step_off), 0, 3 * 1024, 0);
    }
  };
  // Side 1, once its part of V tile t has landed, where some row does not see the whole tile: infinite and NaN values would
  // give NaN with that row's weights of 0. They become 0, and the end of the unit adds them to the rows that see them.
  const auto clean = [&](int t, int buf) __attribute__((always_inline)) {
    if (side == 0 || f_first - t * kTile >= kTile - 1) return;
    __builtin_amdgcn_s_waitcnt(kVmcntLgkm0);
    asm volatile("" ::: "memory");
    float sum = 0.f;
    char* part = lds.v[0] + buf * kTileBytes + wl * 32 * 256 + again(lane) * 16;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(part + i * 1024);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t two = v[e];
        sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, two), bf16x2_t{(__bf16)0.f, (__bf16)0.f}, sum, false);
      }
    }
    const int any = __any(sum != 0.f);
    if (lane == 0) lds.odd[buf][wl] = any;
    if (any) {
#pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        u32x4_t v = *reinterpret_cast<const u32x4_t*>(part + i * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] &= ((v[e] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((v[e] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
        *reinterpret_cast<u32x4_t*>(part + i * 1024) = v;
      }
    }
  };

  // LDS read offsets. K: key 32 t + l32, slot 2 c + half: k_rd ^ 32 c. V: transposing reads of rows 32 t + 16 c2 + 8 a +
  // 4 half + i / 4 and columns 32 dt + 16 g16 + 4 (i % 4), with i = lane % 16 and g16 = (lane / 16) % 2: v_rd ^ 64 dt.
  const int k_rd = l32 * 256 + ((half ^ (l32 & 15)) << 4);
  const int li = lane & 15;
  const int v_rd = (4 * half + (li >> 2)) * 256 + (((2 * ((lane >> 4) & 1) + ((li & 3) >> 1)) ^ ((li >> 2) << 2)) << 4) +
                   8 * (li & 1);

  // This lane's row of unit u: token and head (behind the unit's last token: that one again, which is not stored).
  const auto row_of = [&](const Unit<I>& u, int x, int& tok, int& head) __attribute__((always_inline)) -> int {
    const int heads = heads_of(P, u.hp), tokens = min(P.T, u.S.w - u.j * P.T);
    const int packed = lds.row[x];
    tok = packed >> 16;
    head = packed & 0xffff;
    if (heads != P.GP) {  // the last part of a large group
      tok = x / heads;
      head = x - tok * heads;
    }
    head += u.g * P.G + u.hp * P.GP;
    const bool real = tok < tokens;
    tok = u.j * P.T + min(tok, tokens - 1);
    return real;
  };
  bf16x8_t qf[8];
  int pos;  // of the lane's row
  const auto load_q = [&](const Unit<I>& u) __attribute__((always_inline)) {
    int tok, head;
    const int ln = again(lane);
    row_of(u, w * 32 + (ln & 31), tok, head);
    pos = u.S.len - u.S.w + tok;
    const uint16_t* qp = P.q + (size_t)(u.row0 + tok) * P.q_stride + (size_t)head * kHeadDim + 8 * (ln >> 5);
#pragma unroll
    for (int c = 0; c < 8; ++c) qf[c] = as_bf16x8(ldg16(qp + 16 * c));
  };

  // Side 0: the unit behind that in place `slot`, and its first pages, for both sides. A range's last unit has one of no tiles
  // behind it. In front of a unit's tiles: looked for at its last tile by either side, the next unit held up the barrier by
  // 5,000 cycles a side (19 prompts 774 us, now 757), and inside the loop over the tiles that code slows the loop down (4K tokens over 64K
  // 3.92 ms, now 3.86).
  int slot = 0;
  const auto prepare = [&]() __attribute__((always_inline)) {
    Unit<I> N = get<I>(lds.unit[wl][slot & 3], P);
    if (!advance(N, uniform((I)lds.range[0]), uniform((I)lds.range[1]))) N.t1 = 0;
    put(lds.unit[wl][(slot + 1) & 3], N);
    if (N.t1 == 0) return;
    int e[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) e[r] = page_of(P.table + (size_t)N.n * P.max_pages, uniform(N.S.keys(N.j)), 0, r);
#pragma unroll
    for (int r = 0; r < 2; ++r) lds.pages[wl][r][again(lane)] = e[r];
  };

  int buf = 0;
  if (side == 0) put(lds.unit[wl][0], D);
  fetch_from(D);
  look_up(D.t0);
  load_q(D);
  copy(D.t0, 0, 0);
  clean(D.t0, 0);
  end_phase(true);
  if (side == 1) end_phase(false);

  for (;; ++slot) {
    const Unit<I> D = get<I>(lds.unit[wl][slot & 3], P);
    const bool live = w * 32 < min(P.T, D.S.w - D.j * P.T) * heads_of(P, D.hp);
    const int pos_low = uniform(pos);  // of the wave's rows
    const int pos_top = __builtin_amdgcn_readlane(pos, 31);
    f32x16_t o[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
    // Running maximum of the raw logits, the same in both halves, and this half's share of the sum. A weight is exp2(s c -
    // ref) with ref the rounded m c: one fma, and the rounding is the same factor for all of a row's weights. Where |ref|
    // is large, that factor would be far from 1 (above 2^31, infinity or 0): from then on the wave takes exp2((s - m) c).
    float m = -INFINITY, lsum = 0.f;
    bool far = false;
    int odd_from = INT_MAX;  // first key of the first tile that was cleaned
    const int first_pos = D.S.len - D.S.w + D.j * P.T;

    // What QK hands to PV of the same tile.
    struct Logits {
      f32x16_t s[kKeyTiles];
      float mnew;
      bool on;    // the wave sees something of the tile
      bool edge;  // and some of its rows not all of it
    };
    const auto qk_half = [&](int t, Logits& X) __attribute__((always_inline)) {
      const int key0 = t * kTile;
      auto& s = X.s;
      X.on = live && key0 <= pos_top;
      X.edge = pos_low - key0 < kTile - 1;
      if (!X.on) return;
#pragma unroll
      for (int tt = 0; tt < kKeyTiles; ++tt)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[tt][r] = 0.f;
      int kr = k_rd;
      asm volatile("" : "+v"(kr));  // the chunks' offsets are formed here, not held in registers
      const char* Kb = lds.k[0] + buf * kTileBytes;
      bf16x8_t kf[2][kKeyTiles];
#pragma unroll
      for (int tt = 0; tt < kKeyTiles; ++tt)
        kf[0][tt] = as_bf16x8(*reinterpret_cast<const u32x4_t*>(Kb + kr + tt * 32 * 256));
      __builtin_amdgcn_sched_group_barrier(0x100, kKeyTiles, 0);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        if (c + 1 < 8) {
#pragma unroll
          for (int tt = 0; tt < kKeyTiles; ++tt)
            kf[(c + 1) & 1][tt] = as_bf16x8(*reinterpret_cast<const u32x4_t*>(Kb + (kr ^ (32 * (c + 1))) + tt * 32 * 256));
        }
#pragma unroll
        for (int tt = 0; tt < kKeyTiles; ++tt) s[tt] = mfma32x32x16(kf[c & 1][tt], qf[c], s[tt]);
        if (c + 1 < 8) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, kKeyTiles, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, kKeyTiles - 1, 0);
        } else {
          __builtin_amdgcn_sched_group_barrier(0x008, kKeyTiles, 0);
        }
      }
      if (X.edge) {  // keys behind the row's token (and the zeros behind the last key): -inf, bit by bit
        int qh = pos - key0 - 4 * half;
        asm volatile("" : "+v"(qh));
#pragma unroll
        for (int tt = 0; tt < kKeyTiles; ++tt)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            int d = qh - (32 * tt + 8 * (r >> 2) + (r & 3));
            asm volatile("" : "+v"(d));
            const uint32_t masked = (uint32_t)(d >> 31);
            const float sv = s[tt][r];
            const uint32_t bits = __builtin_bit_cast(uint32_t, sv);
            s[tt][r] = __builtin_bit_cast(float, (bits & ~masked) | (0xFF800000u & masked));
          }
      }
      float mloc = -INFINITY;
#pragma unroll
      for (int tt = 0; tt < kKeyTiles; ++tt)
#pragma unroll
        for (int r = 0; r < 16; ++r) mloc = fmaxf(mloc, s[tt][r]);
      X.mnew = fmaxf(m, half_max(mloc));
    };

    const auto pv_half = [&](Logits& X) __attribute__((always_inline)) {
      if (!X.on) return;
      auto& s = X.s;
      const float mnew = X.mnew;
      __builtin_amdgcn_s_setprio(1);
      const float base = mnew == -INFINITY ? 0.f : mnew;
      float ref = rounded(base, P.scale_log2);
      float alpha = __builtin_amdgcn_exp2f(rounded(m, P.scale_log2) - ref);
      if (far || __any(fabsf(ref) > kFar)) {
        alpha = __builtin_amdgcn_exp2f((m - base) * P.scale_log2);
        if (!far && m != -INFINITY) alpha *= exact_by(m, P.scale_log2);
        far = true;
#pragma unroll
        for (int tt = 0; tt < kKeyTiles; ++tt)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[tt][r] -= base;
        ref = 0.f;
      }
      m = mnew;
      if (__any(alpha != 1.f)) {
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
      }
      constexpr int KC = kTile / 16;
      bf16x8_t pf[KC];
      float rs = 0.f;
#pragma unroll
      for (int kc = 0; kc < KC; ++kc)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float pv = __builtin_amdgcn_exp2f(fmaf(s[kc >> 1][8 * (kc & 1) + e], P.scale_log2, -ref));
          rs += pv;
          pf[kc][e] = (__bf16)pv;
        }
      lsum = fmaf(lsum, alpha, rs);
      const int v_at = (int)(size_t)COSA_LDS(lds.v[0]) + buf * kTileBytes + v_rd;
      int va[4];
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) va[dt] = v_at ^ (64 * dt);
      // Issued directly, so that the offsets go into the instruction; the wait names the fragments, which hands them to
      // the MFMAs and keeps their registers reserved until the data has landed.
      s16x4_t lo[2][4], hi[2][4];
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(lo[0][dt]) : "v"(va[dt]), "i"(0));
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(hi[0][dt]) : "v"(va[dt]), "i"(8 * 256));
      }
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) {
        const int c = kc & 1, nx = c ^ 1;
        asm volatile("s_waitcnt lgkmcnt(0)"
                     : "+v"(lo[c][0]), "+v"(lo[c][1]), "+v"(lo[c][2]), "+v"(lo[c][3]), "+v"(hi[c][0]), "+v"(hi[c][1]),
                       "+v"(hi[c][2]), "+v"(hi[c][3]));
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
          o[dt] = mfma32x32x16(
              __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo[c][dt], hi[c][dt], 0, 1, 2, 3, 4, 5, 6, 7)), pf[kc], o[dt]);
        if (kc + 1 < KC) {
#pragma unroll
          for (int dt = 0; dt < 4; ++dt) {
            asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(lo[nx][dt]) : "v"(va[dt]), "i"((kc + 1) * 16 * 256));
            asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2"
                         : "=v"(hi[nx][dt]) : "v"(va[dt]), "i"((kc + 1) * 16 * 256 + 8 * 256));
          }
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);  // the chunk's MFMAs ...
        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);  // ... then the next chunk's reads
      }
      __builtin_amdgcn_s_setprio(0);
    };

    // Tile t: QK, fetch the next tile (of this unit or of the next one) into the other buffers, barrier, PV, barrier. A
    // wave waits for its own copies at the end of its PV half, a barrier before the other side or it itself reads them.
    bool more = false;
    int i = 0;  // tiles behind the last look_up
    const int t1 = D.t1;
    if (side == 0) prepare();
    int t_end = t1;
    asm volatile("" : "+s"(t_end));  // a loop of its own: `last` is not taken for its exit
    for (int t = D.t0; t < t_end; ++t) {
      const bool last = t + 1 == t1;
      int to = t + 1;
      if (last) {
        const Unit<I> N = get<I>(lds.unit[wl][(slot + 1) & 3], P);
        more = N.t1 != 0;
        i = 0;
        to = 0;
        if (more) {
          fetch_from(N);
#pragma unroll
          for (int r = 0; r < 2; ++r) pg[r] = lds.pages[wl][r][again(lane)];
        }
      } else if (++i == 64) {
        look_up(to);
        i = 0;
      }
      const bool fetch = !last || more;
      Logits X;
      qk_half(t, X);
      if (last && more) load_q(get<I>(lds.unit[wl][(slot + 1) & 3], P));  // its registers are free from here on
      if (fetch) copy(to, i, buf ^ 1);
      end_phase(false);
      if (first_pos - t * kTile < kTile - 1) {
        const u32x4_t odd = *reinterpret_cast<const u32x4_t*>(lds.odd[buf]);
        if (uniform((int)(odd[0] | odd[1] | odd[2] | odd[3]))) odd_from = min(odd_from, t * kTile);
      }
      pv_half(X);
      if (fetch) clean(to, buf ^ 1);
      end_phase(true);
      buf ^= 1;
    }

    if (!more && side == 0) end_phase(false);  // as many barriers on both sides; side 1 need not wait for these results
    const Unit<I> E = get<I>(lds.unit[wl][slot & 3], P);
    const bool whole = E.t0 == 0 && E.t1 == E.tiles;
    if (live) {
      // Results go to memory in whole rows, through the part of the tile that this wave moves, in the buffer of the unit's last
      // tile: its K when side 0 is done (side 1 has had it), its V when side 1 is. A row's 16-byte slot s lies at s ^ row % 16.
      lsum = half_sum(lsum);
      const int ln = again(lane), hf = ln >> 5, r32 = ln & 31, x = w * 32 + r32;
      int tok, head;
      const int real = row_of(E, x, tok, head);
      char* stage = (side ? lds.v[0] : lds.k[0]) + (buf ^ 1) * kTileBytes + wl * 32 * 256;
      char* mine_row = stage + r32 * 256;
      const int n_real = __builtin_popcountll(__ballot(real)) / 2;  // rows of the wave, the first ones
      const int r4 = ln >> 4, slot = ln & 15;  // of rows 4 i + r4
      // The values that were taken as 0, to the staged rows that see them: elements d0 .. d0 + n - 1, T each. Where the row's
      // logit is -inf, the value's weight is 0, and their product is NaN, as it is in the tiles that all rows see.
      const auto add_odd = [&](auto type, int d0, int n, bool none) __attribute__((always_inline)) {
        using V = decltype(type);
        const int32_t* trow = P.table + (size_t)E.n * P.max_pages;
        const int to = (int)min((int64_t)E.t1 * kTile, (int64_t)E.S.len) - 1;
#pragma unroll 1
        for (int t = odd_from; t <= to; ++t) {
          const int32_t e = ld_uniform(trow + (t >> P.log2_page));
          const uint64_t p = (uint32_t)e < (uint64_t)P.n_pages ? (uint32_t)e : 0u;
          const size_t at = uniform((int64_t)((p * page_bytes + (uint64_t)E.g * head_bytes) / 2 + (size_t)(t & page_mask) * kHeadDim));
          const uint32_t two = reinterpret_cast<const uint32_t*>(P.vc + at)[again(lane)];
          if (!__any((two & 0x7f80u) == 0x7f80u || (two & 0x7f800000u) == 0x7f800000u)) continue;
          const uint16_t* qp = P.q + (size_t)(E.row0 + tok) * P.q_stride + (size_t)head * kHeadDim;
          float logit = 0.f;
#pragma unroll 1
          for (int c = 0; c < kHeadDim; ++c)
            logit = fmaf(__uint_as_float((uint32_t)qp[c] << 16), __uint_as_float((uint32_t)P.kc[at + c] << 16), logit);
          if (t <= E.S.len - E.S.w + tok && !none) {
#pragma unroll 1
            for (int i = again(hf) * (n / 2), i1 = i + n / 2; i < i1; ++i) {
              const uint32_t bits = (uint32_t)P.vc[at + d0 + i] << 16;
              if ((bits & 0x7f800000u) == 0x7f800000u) {
                const int byte = i * (int)sizeof(V);
                V* x = reinterpret_cast<V*>(mine_row + (((byte >> 4) ^ (r32 & 15)) << 4) + (byte & 15));
                *x = (V)((float)*x + (logit == -INFINITY ? NAN : __uint_as_float(bits)));
              }
            }
          }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      };
      if (!whole) {
        float* part = P.part + ((size_t)b * 2 + (E.t0 == 0)) * P.part_rows * kRowFloats;
        const float by = far || m == -INFINITY ? 1.f : exact_by(m, P.scale_log2);
#pragma unroll
        for (int hd = 0; hd < 2; ++hd) {
#pragma unroll
          for (int z = 0; z < 8; ++z) {
            const int dt = 2 * hd + (z >> 2), rg = z & 3;
            *reinterpret_cast<f32x4_t*>(mine_row + (((2 * z + hf) ^ (r32 & 15)) << 4)) =
                by * f32x4_t{o[dt][4 * rg], o[dt][4 * rg + 1], o[dt][4 * rg + 2], o[dt][4 * rg + 3]};
          }
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          if (odd_from != INT_MAX) add_odd(0.f, 64 * hd, 64, false);
          f32x4_t v[8];
#pragma unroll
          for (int z = 0; z < 8; ++z)
            v[z] = *reinterpret_cast<const f32x4_t*>(stage + (4 * z + r4) * 256 + ((slot ^ ((4 * z + r4) & 15)) << 4));
#pragma unroll
          for (int z = 0; z < 8; ++z)
            if (4 * z + r4 < n_real)
              *reinterpret_cast<f32x4_t*>(part + (size_t)(w * 32 + 4 * z + r4) * kHeadDim + 64 * hd + 4 * slot) = v[z];
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
        if (hf == 0 && real) {
          part[(size_t)P.part_rows * kHeadDim + x] = m;
          part[(size_t)P.part_rows * (kHeadDim + 1) + x] = by * lsum;
        }
      } else {
        // nothing to attend to: 0 (a sum that is NaN, from a NaN logit, stays NaN)
        const bool none = lsum == 0.f;
        const float inv = none ? 0.f : 1.f / lsum;
        if (__any(none)) {
#pragma unroll
          for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[dt][r] = none ? 0.f : o[dt][r];
        }
        const int out = (E.row0 + tok) * P.Hq + head;
#pragma unroll
        for (int z = 0; z < 16; ++z) {
          const int dt = z >> 2, rg = z & 3;
          uint32_t two[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const __bf16 lo = (__bf16)(o[dt][4 * rg + 2 * e] * inv), hi = (__bf16)(o[dt][4 * rg + 2 * e + 1] * inv);
            two[e] = (uint32_t)__builtin_bit_cast(uint16_t, lo) | ((uint32_t)__builtin_bit_cast(uint16_t, hi) << 16);
          }
          *reinterpret_cast<u32x2_t*>(mine_row + ((z ^ (r32 & 15)) << 4) + 8 * hf) = u32x2_t{two[0], two[1]};
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (odd_from != INT_MAX) add_odd((__bf16)0.f, 0, kHeadDim, none);
        u32x4_t v[8];
        int to[8];
#pragma unroll
        for (int z = 0; z < 8; ++z) {
          v[z] = *reinterpret_cast<const u32x4_t*>(stage + (4 * z + r4) * 256 + ((slot ^ ((4 * z + r4) & 15)) << 4));
          to[z] = __shfl(out, 4 * z + r4, 64);
        }
#pragma unroll
        for (int z = 0; z < 8; ++z)
          if (4 * z + r4 < n_real) *reinterpret_cast<u32x4_t*>(P.o + (size_t)to[z] * kHeadDim + slot * 8) = v[z];
        if (P.lse && hf == 0 && real) P.lse[out] = none ? -INFINITY : (far ? m * P.scale : rounded(m, P.scale_log2) * kLn2) + logf(lsum);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the buffer is free for this wave's next copy
    }
    if (threadIdx.x == 0 && E.t0 > 0 && E.t1 < E.tiles) P.rec[b] = int4{(int)(E.at / (I)lds.range[2]), -1, 0, 0};
    if (threadIdx.x == 0 && E.t0 == 0 && !whole)
      P.rec[b] = int4{E.row0 + E.j * P.T, min(P.T, E.S.w - E.j * P.T) * heads_of(P, E.hp), E.g * P.parts + E.hp,
                      (int)((E.at + (I)(E.tiles - 1) * kChunkTile * E.S.key_slots(E.j)) / (I)lds.range[2])};
    if (!more) break;
  }
}

constexpr int kJoinThreads = 512;
// With 16, 8 rows over 4K tokens, 16 parts, take 22.4 us instead of 19.4, and 128 rows 53 instead of 42; with 3, few workgroups
// join many rows one by one (16 rows over 1000 tokens 25 us instead of 16, 512 over 8K 120 instead of 94).
constexpr int kFewParts = 8;

// Joins the partial results of the unit that begins in range blockIdx.x and ends in another one, for 16 R of its rows: 32
// lanes take R of them. Two where a call has many (128 rows over 4K tokens 41.8 us, 46.2 with one), one where the parts
// are what is many (8 rows over 4K 18.8 us, 20.5 with two). Of a unit of more than kFewParts parts a workgroup takes a row at a
// time, 32 lanes a sixteenth of its parts, and the workgroups of the ranges inside it take rows as well: 2 rows of 20 heads
// over 49K tokens, 193 parts, 24 us instead of 90; 128 rows over 4K 42 instead of 54. Bound: the partial results once, 132 KB a
// unit's range, most of them in the caches (2.7 to 4.0 us for the smallest calls, 14 to 17 for the large ones' 68 MB).
template <int R>
__global__ __launch_bounds__(kJoinThreads) void chunk_join_kernel(const ChunkParams P) {
  int4 rec = P.rec[blockIdx.x];
  if (rec.y == 0) return;
  const int first = rec.y < 0 ? rec.x : (int)blockIdx.x;
  if (rec.y < 0) rec = P.rec[first];
  const int n_parts = rec.w - first + 1;
  const size_t stride = (size_t)P.part_rows * kRowFloats;
  const auto part = [&](int i) { return P.part + ((size_t)(first + i) * 2 + (i == 0)) * stride; };
  const int hp = rec.z % P.parts, heads = heads_of(P, hp), head0 = rec.z / P.parts * P.G + hp * P.GP;
  const int group = threadIdx.x >> 5, t = threadIdx.x & 31;
  const auto join = [&](float& M, float& L, f32x4_t& O, float m, float l, const f32x4_t& o) __attribute__((always_inline)) {
    const float mx = fmaxf(M, m), base = mx == -INFINITY ? 0.f : mx;
    const float a = __builtin_amdgcn_exp2f((M - base) * P.scale_log2);
    const float c = __builtin_amdgcn_exp2f((m - base) * P.scale_log2);
    L = a * L + c * l;
    O = a * O + c * o;
    M = mx;
  };
  // Parts i0, i0 + step ... to rows x: N of them at a time, so that their loads wait side by side.
  const auto add = [&](auto nc, auto rc, const int* x, int i0, int step, float* M, float* L, f32x4_t* O) __attribute__((always_inline)) {
    constexpr int N = decltype(nc)::value, RR = decltype(rc)::value;
    float m[N][RR], l[N][RR];
    f32x4_t o[N][RR];
#pragma unroll
    for (int i = 0; i < N; ++i) {  // behind the last part: that one again, without weight
      const float* p = part(min(i0 + i * step, n_parts - 1));
#pragma unroll
      for (int r = 0; r < RR; ++r) {
        m[i][r] = p[(size_t)P.part_rows * kHeadDim + x[r]];
        l[i][r] = p[(size_t)P.part_rows * (kHeadDim + 1) + x[r]];
        o[i][r] = *reinterpret_cast<const f32x4_t*>(p + (size_t)x[r] * kHeadDim + t * 4);
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i0 + i * step >= n_parts) break;
#pragma unroll
      for (int r = 0; r < RR; ++r) join(M[r], L[r], O[r], m[i][r], l[i][r], o[i][r]);
    }
  };
  const auto write = [&](int x, float M, float L, const f32x4_t& O) __attribute__((always_inline)) {
    const int tok = x / heads;
    const size_t out = (size_t)(rec.x + tok) * P.Hq + head0 + (x - tok * heads);
    const bool none = L == 0.f;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = none ? 0.f : O[e] / L;
    store4(P.o + out * kHeadDim + t * 4, v);
    if (P.lse && t == 0) P.lse[out] = none ? -INFINITY : M * P.scale + logf(L);
  };
  constexpr int kStep = kJoinThreads / 32;
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  const std::integral_constant<int, 8> eight;
  if (n_parts > kFewParts) {
    __shared__ f32x4_t sums[kStep][32];
    __shared__ float tops[kStep], totals[kStep];
    const int workers = (rec.w - first) * gridDim.y;
    for (int x = (blockIdx.x - first) * gridDim.y + blockIdx.y; x < rec.y; x += workers) {
      float M = -INFINITY, L = 0.f;
      f32x4_t O = {0.f, 0.f, 0.f, 0.f};
      if (n_parts <= 2 * kStep) add(two, one, &x, group, kStep, &M, &L, &O);
      else
        for (int i0 = group; i0 < n_parts; i0 += 8 * kStep) add(eight, one, &x, i0, kStep, &M, &L, &O);
      sums[group][t] = O;
      if (t == 0) {
        tops[group] = M;
        totals[group] = L;
      }
      __syncthreads();
      if (group == 0) {
#pragma unroll
        for (int i = 1; i < kStep; ++i) join(M, L, O, tops[i], totals[i], sums[i][t]);
        write(x, M, L, O);
      }
      __syncthreads();
    }
    return;
  }
  const int x0 = blockIdx.y * (kStep * R) + group, last = rec.y - 1;
  if (first != (int)blockIdx.x || x0 > last) return;
  int x[R];
  float M[R], L[R];
  f32x4_t O[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    x[r] = min(x0 + r * kStep, last);
    M[r] = -INFINITY;
    L[r] = 0.f;
    O[r] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const std::integral_constant<int, R> rows;
  if (n_parts <= 2) add(two, rows, x, 0, 1, M, L, O);
  else
    for (int i0 = 0; i0 < n_parts; i0 += 8) add(eight, rows, x, i0, 1, M, L, O);
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (x0 + r * kStep <= last) write(x[r], M[r], L[r], O[r]);
}

// Rows of a partial result: those that a unit can have, an even number, so that every partial result starts at a multiple of 16
// bytes, which the vector loads and stores of O take for granted.
int part_rows(const ChunkShape& sh) {
  const long long rows = std::min<long long>(kChunkRows, (long long)std::min(sh.n_rows, chunk_tokens(sh.G)) * chunk_heads(sh.G));
  return (int)(rows + rows % 2);
}
static_assert(2 * kRowFloats * sizeof(float) % 16 == 0 && kChunkRows % 2 == 0 && kGrid * sizeof(int4) % 16 == 0,
              "partial results lie at multiples of 16 bytes");

}  // namespace

size_t chunk_workspace_bytes(const ChunkShape& sh) {
  return kGrid * sizeof(int4) + (size_t)kGrid * 2 * part_rows(sh) * kRowFloats * sizeof(float);
}

hipError_t launch_chunk_attention(const ChunkShape& sh, const ChunkArgs& a, hipStream_t stream) {
  int4* rec = static_cast<int4*>(a.workspace);
  float* part = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + kGrid * sizeof(int4));
  const int rows = part_rows(sh), T = chunk_tokens(sh.G), parts = chunk_parts(sh.G);
  // Ranges that the rows can make (a power of two of them): units of at most the table's tokens, at least one row each.
  const long long units = std::min<long long>(sh.n_rows, (long long)sh.n_rows / T + sh.B) * sh.Hkv * parts;
  const double ranges = (double)units * ((double)sh.cap() + kUnitKeys) * kFullSlots / kShortest;
  int log2_grid = kLog2Grid;
  while (log2_grid > 3 && ranges <= (double)(1 << (log2_grid - 1))) --log2_grid;
  const int grid = 1 << log2_grid;  // whole rounds over the XCDs
  const ChunkParams P{a.q, a.k_cache, a.v_cache, a.table, a.seq_lens, a.cu_new, part, rec, a.o, a.lse,
                      sh.B, sh.Hq, sh.Hkv, sh.G, chunk_heads(sh.G), parts, T,
                      sh.max_pages, sh.log2_page, sh.n_rows, rows, log2_grid, sh.q_stride, sh.n_pages,
                      sh.scale, std::min(sh.scale * 1.4426950408889634f, FLT_MAX)};  // 0 times infinity is no logit
  if (chunk_narrow(sh.B, sh.n_rows, sh.cap(), (long long)sh.Hkv * parts, T))
    hipLaunchKernelGGL(chunk_kernel<int32_t>, dim3(grid), dim3(kThreads), 0, stream, P);
  else
    hipLaunchKernelGGL(chunk_kernel<int64_t>, dim3(grid), dim3(kThreads), 0, stream, P);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const auto join = [&](auto kernel, int r) {
    const int per = kJoinThreads / 32 * r;
    hipLaunchKernelGGL(kernel, dim3(grid, (rows + per - 1) / per), dim3(kJoinThreads), 0, stream, P);
  };
  if (rows > 64) join(chunk_join_kernel<2>, 2);
  else join(chunk_join_kernel<1>, 1);
  return hipGetLastError();
}

}  // namespace cosa
