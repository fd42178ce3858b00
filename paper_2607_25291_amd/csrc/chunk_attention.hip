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
#include <float.h>
#include <limits.h>

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
constexpr int kGrid = 256;                        // workgroups that share the line: one a CU
constexpr int kShortest = 256;                    // slots of the shortest range
constexpr int kRowFloats = kHeadDim + 2;          // of a partial result: O, maximum, sum

// Partial results of workgroup b: slot 2 b of its first unit, which began in a range before, 2 b + 1 of its last one.
struct ChunkParams {
  const uint16_t *q, *kc, *vc;
  const int32_t *table, *seq_lens, *cu_new;
  float* part;
  int4* rec;  // [kGrid]: a unit that begins in range b and ends in another one: sequence, head and part, unit, last range
  uint16_t* o;
  float* lse;
  int B, Hq, Hkv, G, GP, parts, T;  // GP: heads of a unit
  int max_pages, log2_page, n_rows, part_rows, grid;
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
  return {min(max(len, 0), P.max_pages << P.log2_page), end - row0, P.T};
}
__device__ __forceinline__ ChunkSeq seq_of(const ChunkParams& P, int n) {
  int row0;
  return seq_of(P, P.cu_new[n], P.cu_new[n + 1], P.seq_lens[n], row0);
}

// Uniform reads of data that the kernels never write, through the constant address space: scalar loads.
__device__ __forceinline__ int32_t ld_uniform(const int32_t* p) {
  return *(const __attribute__((address_space(4))) int32_t*)(size_t)p;
}
__device__ __forceinline__ ChunkSeq seq_of_uniform(const ChunkParams& P, int n, int& row0) {
  return seq_of(P, ld_uniform(P.cu_new + n), ld_uniform(P.cu_new + n + 1), ld_uniform(P.seq_lens + n), row0);
}
// Values that are the same in every lane, in scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)x) | (int64_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32;
}

// Heads of unit part hp of a group, its first head, and the rows of unit j.
__device__ __forceinline__ int heads_of(const ChunkParams& P, int hp) { return min(P.G - hp * P.GP, P.GP); }

__device__ __forceinline__ void store8(uint16_t* to, const float (&x)[4], float by) {
  uint32_t w[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const __bf16 lo = (__bf16)(x[2 * e] * by), hi = (__bf16)(x[2 * e + 1] * by);
    w[e] = (uint32_t)__builtin_bit_cast(uint16_t, lo) | ((uint32_t)__builtin_bit_cast(uint16_t, hi) << 16);
  }
  *reinterpret_cast<u32x2_t*>(to) = u32x2_t{w[0], w[1]};
}

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
};

// Tiles [t0, t1) of unit j of sequence n; the result goes to o and lse (part == nullptr) or to part.
__device__ __forceinline__ void walk(const ChunkParams& P, Lds& lds, const ChunkSeq& S, int n, int row0, int g, int hp, int j,
                                     int t0, int t1, float* part) {
  const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int side = w >> 2, wl = w & 3;  // waves w and w + 4 share a SIMD; side 1 runs one phase behind
  const int heads = heads_of(P, hp);
  const int first = j * P.T;  // first token
  const int rows = uniform(min(P.T, S.w - first) * heads);
  const int keys = uniform(S.keys(j));

  // This lane's row (behind the unit's last one: that one again, which is not stored).
  const int xr = min(w * 32 + l32, rows - 1), tok = xr / heads;
  const int row = row0 + first + tok, h = g * P.G + hp * P.GP + (xr - tok * heads);
  const int pos = S.len - S.w + first + tok;
  const int pos_low = __builtin_amdgcn_readfirstlane(pos);                                  // of the wave's rows
  const int pos_top = __builtin_amdgcn_readlane(pos, 31);
  const bool live = w * 32 < rows;

  bf16x8_t qf[8];
  {
    const uint16_t* qp = P.q + (size_t)row * P.q_stride + (size_t)h * kHeadDim + 8 * half;
#pragma unroll
    for (int c = 0; c < 8; ++c) qf[c] = as_bf16x8(ldg16(qp + 16 * c));
  }

  // Copies. Side 0 moves K, side 1 V: wave wl rows 32 wl .. 32 wl + 31 of a tile, in two runs of 16. A lane fills slot
  // lane % 16 of row lane / 16 of four rows with the slot that the layout puts there (K: slot ^ row % 16, V: slot ^ 4 (row %
  // 4), as the MFMA operand and the transposing reads want them).
  const uint64_t head_bytes = (uint64_t)(kHeadDim * 2) << P.log2_page;
  const uint64_t page_bytes = head_bytes * (uint64_t)P.Hkv;
  const uint64_t cache = (uint64_t)uniform((int64_t)((uint64_t)(side ? P.vc : P.kc) + (uint64_t)g * head_bytes));
  const int page_mask = (1 << P.log2_page) - 1;
  const int32_t* trow = P.table + (size_t)n * P.max_pages;
  const int vk = (lane >> 4) * 256 + (((lane & 15) ^ (lane >> 4)) << 4);
  const int vv = (lane >> 4) * 256 + (((lane & 15) ^ ((lane >> 4) << 2)) << 4);
  int pg[2];
  // Physical pages of the runs of tiles t .. t + 63, one tile a lane (run r: rows 32 wl + 16 r).
  auto look_up = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int64_t at = (int64_t)(t + lane) * kTile + wl * 32 + r * 16;
      int p = 0;
      if (at < keys) p = trow[at >> P.log2_page];
      pg[r] = (uint32_t)p < (uint64_t)P.n_pages ? p : 0;
    }
  };
  auto copy = [&](auto is_k, int t, int i, char* dst) __attribute__((always_inline)) {
    constexpr bool IS_K = decltype(is_k)::value;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int at = t * kTile + wl * 32 + r * 16;  // below 2^31 + 128 where it holds a key
      const int valid = uniform(min(max(keys - at, 0), 16));
      const uint64_t p = (uint32_t)__builtin_amdgcn_readlane(pg[r], i & 63);
      const uint64_t base = cache + p * page_bytes + (uint64_t)(at & page_mask) * (kHeadDim * 2);
      const __amdgpu_buffer_rsrc_t rs =
          __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, valid * (kHeadDim * 2), 0x00020000);
      const auto to = COSA_LDS(dst + (wl * 32 + r * 16) * 256);
      // the immediate offset counts for the bounds and moves both addresses
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, to, 16, IS_K ? vk : vv, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, to, 16, IS_K ? vk ^ 64 : vv, 0, 1024, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, to, 16, IS_K ? vk ^ 128 : vv, 0, 2048, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, to, 16, IS_K ? vk ^ 192 : vv, 0, 3072, 0);
    }
  };

  f32x16_t o[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
  float m = -INFINITY;  // running maximum of the raw logits, the same in both halves
  float lsum = 0.f;     // this half's share of the sum

  // LDS read offsets. K: key 32 t + l32, slot 2 c + half: k_rd ^ 32 c. V: transposing reads of rows 32 t + 16 c2 + 8 a +
  // 4 half + i / 4 and columns 32 dt + 16 g16 + 4 (i % 4), with i = lane % 16 and g16 = (lane / 16) % 2: v_rd ^ 64 dt.
  const int k_rd = l32 * 256 + ((half ^ (l32 & 15)) << 4);
  const int li = lane & 15;
  const int v_rd = (4 * half + (li >> 2)) * 256 + (((2 * ((lane >> 4) & 1) + ((li & 3) >> 1)) ^ ((li >> 2) << 2)) << 4) +
                   8 * (li & 1);

  // First key of the rest that finish() takes: from the first tile on that holds an infinite or NaN value which some
  // row does not see, where 0 times it would be NaN.
  int rest = INT_MAX;
  // What QK hands to PV of the same tile.
  struct Logits {
    f32x16_t s[kKeyTiles];
    float mnew;
    bool on;    // the wave sees something of the tile
    bool edge;  // and some of its rows not all of it
    int key0;
  };
  auto qk_half = [&](int t, auto bufc, Logits& X) __attribute__((always_inline)) {
    const char* Kb = lds.k[decltype(bufc)::value];
    const int key0 = t * kTile;
    auto& s = X.s;
    X.key0 = key0;
    X.on = live && key0 <= pos_top && rest == INT_MAX;
    X.edge = pos_low - key0 < kTile - 1;
    if (!X.on) return;
#pragma unroll
    for (int tt = 0; tt < kKeyTiles; ++tt)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[tt][r] = 0.f;
    int kr = k_rd;
    asm volatile("" : "+v"(kr));  // the chunks' offsets are formed here, not held in registers
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

  auto odd_values = [&](const char* Vb) __attribute__((always_inline)) -> bool {
    float sum = 0.f;
#pragma unroll 4
    for (int i = 0; i < kTileBytes / 1024; ++i) {
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(Vb + i * 1024 + lane * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t two = v[e];
        sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, two), bf16x2_t{(__bf16)0.f, (__bf16)0.f}, sum, false);
      }
    }
    return __any(sum != 0.f);
  };
  auto pv_half = [&](auto bufc, const Logits& X) __attribute__((always_inline)) {
    if (!X.on) return;
    const auto& s = X.s;
    const float mnew = X.mnew;
    const char* Vb = lds.v[decltype(bufc)::value];
    if (X.edge && odd_values(Vb)) {
      rest = X.key0;
      return;
    }
    __builtin_amdgcn_s_setprio(1);
    // Differences are taken before the scale: a scaled maximum's rounding would be a factor of every weight.
    const float base = mnew == -INFINITY ? 0.f : mnew;
    const float alpha = __builtin_amdgcn_exp2f((m - base) * P.scale_log2);
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
        const float pv = __builtin_amdgcn_exp2f((s[kc >> 1][8 * (kc & 1) + e] - base) * P.scale_log2);
        rs += pv;
        pf[kc][e] = (__bf16)pv;
      }
    lsum = fmaf(lsum, alpha, rs);
    const int v_at = (int)(size_t)COSA_LDS(Vb) + v_rd;
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
      const int b = kc & 1, nx = b ^ 1;
      asm volatile("s_waitcnt lgkmcnt(0)"
                   : "+v"(lo[b][0]), "+v"(lo[b][1]), "+v"(lo[b][2]), "+v"(lo[b][3]), "+v"(hi[b][0]), "+v"(hi[b][1]),
                     "+v"(hi[b][2]), "+v"(hi[b][3]));
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
        o[dt] = mfma32x32x16(__builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo[b][dt], hi[b][dt], 0, 1, 2, 3, 4, 5, 6, 7)),
                             pf[kc], o[dt]);
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

  constexpr std::integral_constant<int, 0> B0{};
  constexpr std::integral_constant<int, 1> B1{};
  int i = 0;  // tiles behind the last look_up
  look_up(t0);
  if (side == 0) copy(std::true_type{}, t0, 0, lds.k[0]);
  else copy(std::false_type{}, t0, 0, lds.v[0]);
  end_phase(true);

  // Tile t in buffers BUF: QK, fetch tile t + 1 into the other buffers, barrier, PV, barrier. A wave waits for its own
  // copies at the end of its PV half, a barrier before the other side or it itself reads them.
  auto tile = [&](int t, auto bufc) __attribute__((always_inline)) {
    constexpr int BUF = decltype(bufc)::value;
    Logits X;
    qk_half(t, bufc, X);
    if (t + 1 < t1) {
      if (++i == 64) {
        look_up(t + 1);
        i = 0;
      }
      if (side == 0) copy(std::true_type{}, t + 1, i, lds.k[BUF ^ 1]);
      else copy(std::false_type{}, t + 1, i, lds.v[BUF ^ 1]);
    }
    end_phase(false);
    pv_half(bufc, X);
    end_phase(true);
  };
  if (side == 1) end_phase(false);
  for (int t = t0; t < t1; t += 2) {
    tile(t, B0);
    if (t + 1 < t1) tile(t + 1, B1);
  }
  if (side == 0) end_phase(false);  // as many barriers on both sides

  // The keys from `rest` on one by one, for values that only some rows see (at most the unit's last tiles).
  const auto finish = [&]() __attribute__((always_inline)) {
    const int to = (int)min((int64_t)t1 * kTile, (int64_t)pos_top + 1);
#pragma unroll 1
    for (int t = rest; t < to; ++t) {
      const int32_t e = ld_uniform(trow + (t >> P.log2_page));
      const uint64_t p = (uint32_t)e < (uint64_t)P.n_pages ? (uint32_t)e : 0u;
      const size_t at = (p * page_bytes + (uint64_t)g * head_bytes) / 2 + (size_t)(t & page_mask) * kHeadDim;
      float dot = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const bf16x8_t k = as_bf16x8(ldg16(P.kc + at + 16 * c + 8 * half));
#pragma unroll
        for (int i = 0; i < 8; ++i) dot = fmaf((float)k[i], (float)qf[c][i], dot);
      }
      const bool sees = t <= pos;
      dot = half_sum(dot);
      const float logit = sees ? dot : -INFINITY;
      const float mn = fmaxf(m, logit), base = mn == -INFINITY ? 0.f : mn;
      const float alpha = __builtin_amdgcn_exp2f((m - base) * P.scale_log2);
      const float pv = __builtin_amdgcn_exp2f((logit - base) * P.scale_log2);
      m = mn;
      lsum = lsum * alpha + (half == 0 ? pv : 0.f);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const u32x2_t v = *reinterpret_cast<const u32x2_t*>(P.vc + at + 8 * i + 4 * half);
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          const float x = __uint_as_float(z & 1 ? v[z >> 1] & 0xffff0000u : v[z >> 1] << 16);
          o[i >> 2][4 * (i & 3) + z] = o[i >> 2][4 * (i & 3) + z] * alpha + (sees ? pv * x : 0.f);
        }
      }
    }
  };
  if (rest != INT_MAX) finish();
  lsum = half_sum(lsum);
  int again = threadIdx.x & 31;
  asm volatile("" : "+v"(again));  // the row is found again here, not held in registers over the walk
  const int x = w * 32 + again;
  if (x < rows) {
    if (part) {
      float* to = part + (size_t)x * kHeadDim;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int rg = 0; rg < 4; ++rg)
          *reinterpret_cast<f32x4_t*>(to + 32 * dt + 8 * rg + 4 * half) =
              f32x4_t{o[dt][4 * rg], o[dt][4 * rg + 1], o[dt][4 * rg + 2], o[dt][4 * rg + 3]};
      if (half == 0) {
        part[(size_t)P.part_rows * kHeadDim + x] = m;
        part[(size_t)P.part_rows * (kHeadDim + 1) + x] = lsum;
      }
    } else {
      // nothing to attend to: 0 (a sum that is NaN, from a NaN logit, stays NaN)
      const int tok = x / heads;
      const size_t out = (size_t)(row0 + first + tok) * P.Hq + g * P.G + hp * P.GP + (x - tok * heads);
      const bool none = lsum == 0.f;
      uint16_t* to = P.o + out * kHeadDim;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int rg = 0; rg < 4; ++rg) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = none ? 0.f : o[dt][4 * rg + e] / lsum;
          store8(to + 32 * dt + 8 * rg + 4 * half, v, 1.f);
        }
      if (P.lse && half == 0) P.lse[out] = none ? -INFINITY : m * P.scale + logf(lsum);
    }
  }
}

__global__ __attribute__((amdgpu_flat_work_group_size(kThreads, kThreads))) __attribute__((amdgpu_waves_per_eu(2, 2)))
void chunk_kernel(const ChunkParams P) {
  __shared__ __attribute__((aligned(1024))) Lds lds;
  __shared__ int64_t sums[kWaves];
  __shared__ int64_t found_at;
  __shared__ int found;
  // Slots of the sequences: every thread a stretch of them.
  const int heads = P.Hkv * P.parts;
  const int per = (P.B + kThreads - 1) / kThreads;
  const int n0 = min((int)threadIdx.x * per, P.B), n1 = min(n0 + per, P.B);
  int64_t mine = 0, total = 0;
  for (int n = n0; n < n1; ++n) mine += seq_of(P, n).slots() * heads;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int64_t at = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up((long long)at, d, 64);
    if (lane >= d) at += y;
  }
  if (lane == 63) sums[w] = at;
  __syncthreads();
  at -= mine;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    if (i < w) at += sums[i];
    total += sums[i];
  }
  total = uniform(total);
  const ChunkRanges R = chunk_ranges(total, P.grid, kShortest);
  // Neighbouring ranges, which mostly share a KV head, go to one XCD.
  if ((int)blockIdx.x >= R.n && threadIdx.x == 0) P.rec[blockIdx.x] = int4{-1, 0, 0, 0};  // no range has this number
  const int per_xcd = (R.n + kNumXcd - 1) / kNumXcd, k = blockIdx.x / kNumXcd;
  const int b = (blockIdx.x % kNumXcd) * per_xcd + k;
  if (k >= per_xcd || b >= R.n) return;
  const int64_t A = b * R.length, end = min(A + R.length, total);
  if (A >= at && A < at + mine) {
    int n = n0;
    for (;; ++n) {
      const int64_t t = seq_of(P, n).slots() * heads;
      if (A < at + t) break;
      at += t;
    }
    found = n;
    found_at = at;
  }
  __syncthreads();
  int n = uniform(found);
  int64_t U = uniform(found_at);
  int row0;
  ChunkSeq S = seq_of_uniform(P, n, row0);
  int64_t one = S.slots();
  int hh = uniform((int)((A - U) / one));
  U += hh * one;
  int j = uniform(S.find(A - U));
  U = uniform(U + S.start(j));
  int4 rec = {-1, 0, 0, 0};
  while (U < end) {
    const int tiles = uniform(S.tiles(j)), t0 = uniform(chunk_tile0(A, U)), t1 = uniform(chunk_tile1(end, U, tiles));
    if (t0 < t1) {
      float* part = nullptr;
      if (t0 > 0 || t1 < tiles) part = P.part + ((size_t)b * 2 + (t0 == 0)) * P.part_rows * kRowFloats;
      if (t0 == 0 && t1 < tiles) rec = {n, hh, j, (int)((U + (int64_t)(tiles - 1) * kChunkTile) / R.length)};
      walk(P, lds, S, n, row0, uniform(hh / P.parts), uniform(hh % P.parts), j, t0, t1, part);
    }
    U = uniform(U + S.keys(j) + kUnitSlots);
    if (U >= end) break;
    if (++j == S.units()) {
      j = 0;
      if (++hh == heads) {
        hh = 0;
        do S = seq_of_uniform(P, ++n, row0); while (S.w == 0);  // there are slots left, so there is one
      }
    }
  }
  if (threadIdx.x == 0) P.rec[b] = rec;
}

constexpr int kJoinRows = 16;  // rows of a workgroup of the join, 32 lanes each

// Joins the partial results of the unit that begins in range blockIdx.x and ends in another one, for kJoinRows of its rows.
__global__ __launch_bounds__(kJoinRows * 32) void chunk_join_kernel(const ChunkParams P) {
  const int4 rec = P.rec[blockIdx.x];
  if (rec.x < 0) return;
  int row0;
  const ChunkSeq S = seq_of_uniform(P, __builtin_amdgcn_readfirstlane(rec.x), row0);
  const int g = rec.y / P.parts, hp = rec.y % P.parts, heads = heads_of(P, hp), first = rec.z * P.T;
  const int x = blockIdx.y * kJoinRows + (threadIdx.x >> 5), t = threadIdx.x & 31;
  if (x >= min(P.T, S.w - first) * heads) return;
  const int tok = x / heads;
  const size_t out = (size_t)(row0 + first + tok) * P.Hq + g * P.G + hp * P.GP + (x - tok * heads);
  const size_t stride = (size_t)P.part_rows * kRowFloats;
  const int n_parts = rec.w - (int)blockIdx.x + 1;
  const auto part = [&](int i) { return P.part + ((size_t)(blockIdx.x + i) * 2 + (i == 0)) * stride; };
  float M = -INFINITY, L = 0.f;
  f32x4_t O = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < n_parts; i0 += 4) {
    float m[4], l[4];
    f32x4_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // behind the last part: that one again, without weight
      const float* p = part(min(i0 + i, n_parts - 1));
      m[i] = p[(size_t)P.part_rows * kHeadDim + x];
      l[i] = p[(size_t)P.part_rows * (kHeadDim + 1) + x];
      o[i] = *reinterpret_cast<const f32x4_t*>(p + (size_t)x * kHeadDim + t * 4);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i0 + i >= n_parts) break;
      const float mx = fmaxf(M, m[i]), base = mx == -INFINITY ? 0.f : mx;
      const float a = __builtin_amdgcn_exp2f((M - base) * P.scale_log2), c = __builtin_amdgcn_exp2f((m[i] - base) * P.scale_log2);
      L = a * L + c * l[i];
      O = a * O + c * o[i];
      M = mx;
    }
  }
  const bool none = L == 0.f;
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = none ? 0.f : O[e] / L;
  store8(P.o + out * kHeadDim + t * 4, v, 1.f);
  if (P.lse && t == 0) P.lse[out] = none ? -INFINITY : M * P.scale + logf(L);
}

// Rows of a partial result: those that a unit can have.
int part_rows(const ChunkShape& sh) {
  return (int)std::min<long long>(kChunkRows, (long long)std::min(sh.n_rows, chunk_tokens(sh.G)) * chunk_heads(sh.G));
}

}  // namespace

size_t chunk_workspace_bytes(const ChunkShape& sh) {
  return kGrid * sizeof(int4) + (size_t)kGrid * 2 * part_rows(sh) * kRowFloats * sizeof(float);
}

hipError_t launch_chunk_attention(const ChunkShape& sh, const ChunkArgs& a, hipStream_t stream) {
  int4* rec = static_cast<int4*>(a.workspace);
  float* part = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + kGrid * sizeof(int4));
  const int rows = part_rows(sh), T = chunk_tokens(sh.G), parts = chunk_parts(sh.G);
  // Ranges that the rows can make: units of at most the table's tokens, at least one row each.
  const long long units = std::min<long long>(sh.n_rows, (long long)sh.n_rows / T + sh.B) * sh.Hkv * parts;
  const double slots = (double)units * ((double)sh.cap() + kUnitSlots);
  const int grid = slots / kShortest + 1 < kGrid ? (int)(slots / kShortest) + 1 : kGrid;
  const ChunkParams P{a.q, a.k_cache, a.v_cache, a.table, a.seq_lens, a.cu_new, part, rec, a.o, a.lse,
                      sh.B, sh.Hq, sh.Hkv, sh.G, chunk_heads(sh.G), parts, T,
                      sh.max_pages, sh.log2_page, sh.n_rows, rows, grid, sh.q_stride, sh.n_pages,
                      sh.scale, std::min(sh.scale * 1.4426950408889634f, FLT_MAX)};  // 0 times infinity is no logit
  // whole rounds over the XCDs, so that every range has its workgroup
  const int wgs = (grid + kNumXcd - 1) / kNumXcd * kNumXcd;
  hipLaunchKernelGGL(chunk_kernel, dim3(wgs), dim3(kThreads), 0, stream, P);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || grid == 1) return e;
  hipLaunchKernelGGL(chunk_join_kernel, dim3(grid, (rows + kJoinRows - 1) / kJoinRows), dim3(kJoinRows * 32), 0, stream, P);
  return hipGetLastError();
}

}  // namespace cosa
