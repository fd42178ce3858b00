// New K and V rows into a paged cache by slot, and the bounds of the keys in the pages they touch, for
// gfx950.
//
// A run is a stretch of rows whose slots follow each other within one page; its rows are contiguous in
// the cache. A wave owns the runs that start in its chunk of rows, for one KV head: 16 lanes move a row
// of 256 bytes, four rows per load, and keep the minimum and maximum of their eight elements. So a
// page's bounds need one wave and no atomics. bf16 values are compared as 16-bit integers (the value's
// bits with the magnitude inverted under a sign), two per instruction.
#include "cosa_device.h"
#include "decode_internal.h"

namespace cosa {
namespace {

typedef int16_t i16x8_t __attribute__((ext_vector_type(8)));

// Order-preserving map between bf16 bits and signed 16-bit integers; its own inverse.
__device__ __forceinline__ i16x8_t ordered(i16x8_t x) { return x ^ ((x >> 15) & (int16_t)0x7fff); }

__device__ __forceinline__ i16x8_t shfl_xor8(i16x8_t x, int d) {
  u32x4_t u = __builtin_bit_cast(u32x4_t, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = (uint32_t)__shfl_xor((int)u[i], d, 64);
  return __builtin_bit_cast(i16x8_t, u);
}

template <bool BOUNDS>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs A, int log2_chunk, long long n_waves) {
  const long long id = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= n_waves) return;
  const int lane = threadIdx.x & 63, r = lane & 15, gq = lane >> 4;
  const int g = (int)(id % A.Hkv);
  const long long t0 = (id / A.Hkv) << log2_chunk;
  const int64_t page = 1ll << A.log2_page, n_slots = (int64_t)A.n_pages << A.log2_page;

  // Rows of the chunk at which a run starts.
  const long long tl = t0 + lane;
  bool start = false;
  if (lane < (1 << log2_chunk) && tl < A.n_tokens) {
    const int64_t s = A.slots[tl];
    start = s >= 0 && s < n_slots && ((s & (page - 1)) == 0 || tl == 0 || A.slots[tl - 1] != s - 1);
  }
  uint64_t starts = __ballot(start);
  while (starts) {
    long long t = t0 + __builtin_ctzll(starts);
    starts &= starts - 1;
    const int64_t s0 = A.slots[t];
    const int off = (int)(s0 & (page - 1));
    const int64_t most = min((int64_t)(page - off), (int64_t)(A.n_tokens - t));  // rows the page and the call have left
    const size_t row = (((size_t)(s0 >> A.log2_page) * A.Hkv + g) << A.log2_page) + off;
    i16x8_t lo, hi;
#pragma unroll
    for (int i = 0; i < 8; ++i) lo[i] = 0x7fff, hi[i] = (int16_t)0x8000;
    int64_t done = 0;
    while (done < most) {
      // rows among the next 64 that continue the run
      const bool here = done + lane < most && A.slots[t + done + lane] == s0 + done + lane;
      const uint64_t same = __ballot(here);
      const int n = ~same ? __builtin_ctzll(~same) : 64;
      for (int i = 0; i < n; i += 4) {
        if (i + gq < n) {
          const long long tt = t + done + i + gq;
          const u32x4_t kk = ldg16(A.k + tt * A.k_stride + g * kHeadDim + r * 8);
          const u32x4_t vv = ldg16(A.v + tt * A.v_stride + g * kHeadDim + r * 8);
          const size_t at = (row + done + i + gq) * kHeadDim + r * 8;
          *reinterpret_cast<u32x4_t*>(A.k_cache + at) = kk;
          *reinterpret_cast<u32x4_t*>(A.v_cache + at) = vv;
          if (BOUNDS) {
            const i16x8_t o = ordered(__builtin_bit_cast(i16x8_t, kk));
            lo = __builtin_elementwise_min(lo, o);
            hi = __builtin_elementwise_max(hi, o);
          }
        }
      }
      done += n;
      if (n < 64) break;
    }
    if (BOUNDS) {
#pragma unroll
      for (int d = 16; d < 64; d <<= 1) {
        lo = __builtin_elementwise_min(lo, shfl_xor8(lo, d));
        hi = __builtin_elementwise_max(hi, shfl_xor8(hi, d));
      }
      if (gq < 2) {
        u32x4_t* b = reinterpret_cast<u32x4_t*>(
            A.bounds + (((size_t)(s0 >> A.log2_page) * A.Hkv + g) * 2 + gq) * kHeadDim + r * 8);
        i16x8_t x = gq ? hi : lo;
        if (off) {
          const i16x8_t old = ordered(__builtin_bit_cast(i16x8_t, *b));
          x = gq ? __builtin_elementwise_max(x, old) : __builtin_elementwise_min(x, old);
        }
        *b = __builtin_bit_cast(u32x4_t, ordered(x));
      }
    }
  }
}

}  // namespace

hipError_t launch_kv_append(const AppendArgs& a, hipStream_t stream) {
  // Rows of a wave's chunk: as many as still leave 4096 waves (four for each of the 1024 SIMDs), so that a decode
  // step's single rows run side by side and a long prompt's pages do not start 16 waves for one run.
  int log2_chunk = 6;
  while (log2_chunk > 0 && ((a.n_tokens + (1 << log2_chunk) - 1) >> log2_chunk) * a.Hkv < 4096) --log2_chunk;
  const long long n_waves = ((a.n_tokens + (1ll << log2_chunk) - 1) >> log2_chunk) * a.Hkv;
  const dim3 grid((unsigned)((n_waves + 3) / 4));
  if (a.bounds) hipLaunchKernelGGL((kv_append_kernel<true>), grid, dim3(256), 0, stream, a, log2_chunk, n_waves);
  else hipLaunchKernelGGL((kv_append_kernel<false>), grid, dim3(256), 0, stream, a, log2_chunk, n_waves);
  return hipGetLastError();
}

}  // namespace cosa
