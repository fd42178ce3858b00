// New K and V rows into a paged cache by slot, and the bounds of the keys in the pages they touch, for
// gfx950.
//
// A run is a stretch of rows whose slots follow each other within one page; its rows are contiguous in
// the cache. A workgroup owns the runs that start in its chunk of rows, for one KV head: its waves take 64
// rows of a run in turn, 16 lanes a row of 256 bytes, and keep the minimum and maximum of their eight
// elements. So a page's bounds need one workgroup and no atomics; it has a wave for every 64 tokens of a
// page (up to 16). bf16 values are compared as 16-bit integers (the value's bits with the magnitude
// inverted under a sign), two per instruction.
//
// Bound: HBM. 35.7K rows of 8 heads (146 MB moved): 26 us, 5.6 TB/s, where a large copy reaches 5.0. With event times:
// stores that the caches do not keep 34.6 us, 42.4 without; four rows of a lane loaded before the first is
// stored 34.6, 36.4 one by one; one wave per workgroup 31.8, four 34.6.
#include <type_traits>

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

template <bool BOUNDS, int NW>
__global__ __launch_bounds__(NW * 64) void kv_append_kernel(AppendArgs A, int log2_chunk) {
  __shared__ uint64_t starts[NW];
  __shared__ i16x8_t part[BOUNDS ? NW : 1][32];
  const int lane = threadIdx.x & 63, r = lane & 15, gq = lane >> 4;
  const int w = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = (int)(blockIdx.x % (unsigned)A.Hkv);
  const long long t0 = (long long)(blockIdx.x / (unsigned)A.Hkv) << log2_chunk;
  const int64_t page = 1ll << A.log2_page, n_slots = (int64_t)A.n_pages << A.log2_page;

  // Rows of the chunk at which a run starts.
  const long long tl = t0 + threadIdx.x;
  bool start = false;
  if ((int)threadIdx.x < (1 << log2_chunk) && tl < A.n_tokens) {
    const int64_t s = A.slots[tl];
    start = s >= 0 && s < n_slots && ((s & (page - 1)) == 0 || tl == 0 || A.slots[tl - 1] != s - 1);
  }
  const uint64_t mine = __ballot(start);
  if (NW > 1) {
    if (lane == 0) starts[w] = mine;
    __syncthreads();
  }
  for (int word = 0; word < NW; ++word) {
    uint64_t left = NW == 1 ? mine : starts[word];
    while (left) {
      const long long t = t0 + word * 64 + __builtin_ctzll(left);
      left &= left - 1;
      const int64_t s0 = A.slots[t];
      const int off = (int)(s0 & (page - 1));
      const int64_t most = min((int64_t)(page - off), (int64_t)(A.n_tokens - t));  // rows the page and the call have left
      const size_t row = (((size_t)(s0 >> A.log2_page) * A.Hkv + g) << A.log2_page) + off;
      i16x8_t lo, hi;
#pragma unroll
      for (int i = 0; i < 8; ++i) lo[i] = 0x7fff, hi[i] = (int16_t)0x8000;
      // Rows i .. i + 4 J - 1 of the n at row `done` of the run; lanes behind n read the last row again, which changes no
      // bound.
      const auto copy = [&](auto J, int64_t done, int i, int n) __attribute__((always_inline)) {
        u32x4_t kk[J], vv[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const long long tt = t + done + min(i + 4 * j + gq, n - 1);
          kk[j] = ldg16(A.k + tt * A.k_stride + g * kHeadDim + r * 8);
          vv[j] = ldg16(A.v + tt * A.v_stride + g * kHeadDim + r * 8);
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const int x = i + 4 * j + gq;
          if (x < n) {
            const size_t at = (row + done + x) * kHeadDim + r * 8;
            __builtin_nontemporal_store(kk[j], reinterpret_cast<u32x4_t*>(A.k_cache + at));
            __builtin_nontemporal_store(vv[j], reinterpret_cast<u32x4_t*>(A.v_cache + at));
          }
          if (BOUNDS) {
            const i16x8_t o = ordered(__builtin_bit_cast(i16x8_t, kk[j]));
            lo = __builtin_elementwise_min(lo, o);
            hi = __builtin_elementwise_max(hi, o);
          }
        }
      };
      for (int64_t done = w * 64; done < most; done += NW * 64) {
        // rows among these 64 that continue the run
        const bool here = done + lane < most && A.slots[t + done + lane] == s0 + done + lane;
        const uint64_t same = __ballot(here);
        const int n = ~same ? __builtin_ctzll(~same) : 64;
        int i = 0;
        for (; i + 4 < n; i += 16) copy(std::integral_constant<int, 4>{}, done, i, n);
        if (i < n) copy(std::integral_constant<int, 1>{}, done, i, n);
        if (n < 64) break;
      }
      if (BOUNDS) {
#pragma unroll
        for (int d = 16; d < 64; d <<= 1) {
          lo = __builtin_elementwise_min(lo, shfl_xor8(lo, d));
          hi = __builtin_elementwise_max(hi, shfl_xor8(hi, d));
        }
        i16x8_t x = gq ? hi : lo;  // of lanes 0 .. 31
        if (NW > 1) {
          if (gq < 2) part[w][lane] = x;
          __syncthreads();
        }
        if (w == 0 && gq < 2) {
          u32x4_t* b = reinterpret_cast<u32x4_t*>(
              A.bounds + (((size_t)(s0 >> A.log2_page) * A.Hkv + g) * 2 + gq) * kHeadDim + r * 8);
#pragma unroll
          for (int i = 1; i < NW; ++i)
            x = gq ? __builtin_elementwise_max(x, part[i][lane]) : __builtin_elementwise_min(x, part[i][lane]);
          if (off) {
            const i16x8_t old = ordered(__builtin_bit_cast(i16x8_t, *b));
            x = gq ? __builtin_elementwise_max(x, old) : __builtin_elementwise_min(x, old);
          }
          *b = __builtin_bit_cast(u32x4_t, ordered(x));
        }
        if (NW > 1) __syncthreads();  // part is used again
      }
    }
  }
}

template <int NW>
hipError_t launch_t(const AppendArgs& a, hipStream_t stream) {
  // Rows of a chunk: a page, or fewer where that leaves less than 4096 waves (four for each of the 1024 SIMDs), so
  // that a decode step's single rows run side by side and a long prompt's pages do not start workgroups
  // that find no run (pages of 16: 114 us for 537 MB, 119 with chunks of 64; pages of 64: 34.6 us for 146 MB, 51.8
  // with chunks of 16).
  int log2_chunk = 0;
  while ((2 << log2_chunk) <= NW * 64 && log2_chunk < a.log2_page &&
         ((a.n_tokens + (2ll << log2_chunk) - 1) >> (log2_chunk + 1)) * a.Hkv * NW >= 4096)
    ++log2_chunk;
  const dim3 grid((unsigned)(((a.n_tokens + (1ll << log2_chunk) - 1) >> log2_chunk) * a.Hkv));
  if (a.bounds) hipLaunchKernelGGL((kv_append_kernel<true, NW>), grid, dim3(NW * 64), 0, stream, a, log2_chunk);
  else hipLaunchKernelGGL((kv_append_kernel<false, NW>), grid, dim3(NW * 64), 0, stream, a, log2_chunk);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_append(const AppendArgs& a, hipStream_t stream) {
  // A wave for every 64 tokens of a page, up to 16: 64K rows in pages of 256 / 2048 114 / 143 us with events, 253 / 962
  // with one wave; single rows in pages of 256 12.4 us, 11.0 with one.
  switch (a.log2_page) {
    case 4: case 5: case 6: return launch_t<1>(a, stream);
    case 7: return launch_t<2>(a, stream);
    case 8: return launch_t<4>(a, stream);
    case 9: return launch_t<8>(a, stream);
    default: return launch_t<16>(a, stream);
  }
}

}  // namespace cosa
