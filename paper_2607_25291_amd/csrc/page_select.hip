// The pages that every KV head keeps of a decode step, for gfx950: one workgroup per (sequence, KV
// head).
//
// The rows' maxima, then one 32-bit key per page in LDS whose order is the order of selection (forced
// pages, NaN, then descending s). A radix selection finds the K-th largest key and how many pages that
// equal it are kept; a scan over the pages then packs the kept ones in ascending order, so the list needs
// no sort.
//
// Bound: latency, the barriers between its steps, and for about a tenth the first digit: the differences span a few
// binary exponents, so their pages crowd into a few tens of its bins. 256 rows of up to 4096 pages, 7 heads: 12.1 us
// for 8.7 MB (events 17.6; 16.0 with differences over 240 exponents, 25.8 with all equal); 8 rows of 256 pages, 4
// heads: 6.0 us, of which an empty launch takes 2. Comparing all pairs of 256 keys instead of the radix selection:
// 14.2 us.
#include <mutex>

#include "cosa_device.h"
#include "decode_internal.h"
#include "select_wave.h"

namespace cosa {
namespace {

constexpr uint32_t kForced = 0xffffffffu, kNan = 0xfffffffeu;

__device__ __forceinline__ uint32_t key_of(float s) {
  const uint32_t b = __float_as_uint(s + 0.f);  // -0 counts as 0
  if ((b & 0x7fffffffu) > 0x7f800000u) return kNan;
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

constexpr int kBins = 2048;

// Scores of kHeads heads from h0 on (the last one again behind G) at pages j, j + T, j + 2 T, j + 3 T (-inf behind the
// row).
template <int T, int kHeads>
__device__ __forceinline__ void load_scores(float (&x)[kHeads][4], const PageSelectArgs& A, const float* score, int h0,
                                            int j, int np) {
#pragma unroll
  for (int k = 0; k < kHeads; ++k) {
    const float* row = score + (size_t)min(h0 + k, A.G - 1) * A.max_pages;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[k][i] = j + i * T < np ? row[j + i * T] : -INFINITY;
  }
}

template <int T, int kHeads>
__global__ __launch_bounds__(T) void page_select_kernel(PageSelectArgs A) {
  constexpr int kWaves = T / 64, kPer = kBins / T;
  extern __shared__ __align__(16) uint32_t lds[];
  uint32_t* keys = lds;                                                       // max_pages, in fours
  float* top = reinterpret_cast<float*>(lds + (A.max_pages + 3) / 4 * 4);     // row maxima of the group's heads, in kHeads
  __shared__ uint32_t hist[3][kBins], waves[kWaves], pick[3];
  __shared__ float part[kHeads][kWaves];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int u = blockIdx.x, n = u / A.Hkv, g = u % A.Hkv;
  const int page = 1 << A.log2_page;
  const int len = min(max(A.seq_lens[n], 0), A.max_pages << A.log2_page);
  const int np = (int)(((unsigned)len + page - 1) >> A.log2_page);
  int32_t* out = A.pages + (size_t)u * A.max_keep;
  const int frac = (int)((A.fraction_micro * np + 999999) / 1000000);
  const int K = min(np, max(A.sink + A.recent, min(A.max_keep, max(A.min_keep, frac))));
  if (threadIdx.x == 0) A.count[u] = K;
  // unsigned: a list may be as wide as 2^31 - 1
  for (uint32_t j = (uint32_t)K + threadIdx.x; j < (uint32_t)A.max_keep; j += T) out[j] = -1;
  if (K == np) {
    for (int j = threadIdx.x; j < K; j += T) out[j] = j;
    return;
  }
  const float* score = A.score + ((size_t)n * A.Hq + (size_t)g * A.G) * A.max_pages;
  for (int i = threadIdx.x; i < kBins; i += T) hist[0][i] = 0;
  // Row maxima, kHeads at a time. Up to so many heads of 4 T pages stay in registers for the keys.
  float x[kHeads][4];
  for (int h0 = 0; h0 < A.G; h0 += kHeads) {
    float m[kHeads];
#pragma unroll
    for (int k = 0; k < kHeads; ++k) m[k] = -INFINITY;
    for (int j = threadIdx.x; j < np; j += 4 * T) {
      load_scores<T, kHeads>(x, A, score, h0, j, np);
#pragma unroll
      for (int k = 0; k < kHeads; ++k) m[k] = fmaxf(m[k], fmaxf(fmaxf(x[k][0], x[k][1]), fmaxf(x[k][2], x[k][3])));
    }
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
      m[k] = wave_max(m[k]);
      if (lane == 0) part[k][w] = m[k];
    }
    __syncthreads();
    if (threadIdx.x < kHeads * 16) {  // 16 lanes a head
      float t = row16_max((int)(threadIdx.x & 15) < kWaves ? part[threadIdx.x >> 4][threadIdx.x & 15] : -INFINITY);
      if ((threadIdx.x & 15) == 0) top[h0 + (threadIdx.x >> 4)] = t;
    }
    __syncthreads();
  }
  const bool kept_in_registers = A.G <= kHeads && np <= 4 * T;
  for (int j = threadIdx.x; j < np; j += 4 * T) {
    float s[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    for (int h0 = 0; h0 < A.G; h0 += kHeads) {
      if (!kept_in_registers) load_scores<T, kHeads>(x, A, score, h0, j, np);
#pragma unroll
      for (int k = 0; k < kHeads; ++k) {
        const float t = top[min(h0 + k, A.G - 1)];
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = vmax(s[i], x[k][i] - t);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int jj = j + i * T;
      if (jj < np) keys[jj] = jj < A.sink || jj >= np - A.recent ? kForced : key_of(s[i]);
    }
  }

  __syncthreads();

  // The K-th largest key by its digits of 11, 11 and 10 bits; it ends early where a digit's pages are all kept.
  uint32_t prefix = 0, mask = 0, want = (uint32_t)K;
  bool whole = false;
#pragma unroll
  for (int pass = 0; pass < 3 && !whole; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t digits = pass == 2 ? 1023u : 2047u;
    for (int j = threadIdx.x; j < np; j += T) {
      const uint32_t k = keys[j];
      if ((k & mask) == prefix) atomicAdd(&hist[pass][(k >> shift) & digits], 1u);
    }
    __syncthreads();
    if (pass < 2)
      for (int i = threadIdx.x; i < kBins; i += T) hist[pass + 1][i] = 0;
    // Thread t counts bins from the largest digit down: kBins - 1 - t kPer, ...
    uint32_t c[kPer], s = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) s += c[i] = hist[pass][kBins - 1 - (int)threadIdx.x * kPer - i];
    const uint32_t incl = wave_incl_scan(s, lane);
    if (lane == 63) waves[w] = incl;
    __syncthreads();
    uint32_t before = incl - s;
#pragma unroll
    for (int i = 0; i < kWaves; ++i)
      if (i < w) before += waves[i];
    if (before < want && before + s >= want) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (before < want && before + c[i] >= want) {
          pick[0] = (uint32_t)(kBins - 1 - (int)threadIdx.x * kPer - i);
          pick[1] = want - before;
          pick[2] = c[i];
        }
        before += c[i];
      }
    }
    __syncthreads();
    prefix |= pick[0] << shift;
    mask |= digits << shift;
    want = pick[1];
    whole = want == pick[2];
  }

  // Kept: keys above the prefix, and of those that share it all (whole) or the first `want` pages.
  uint32_t kept = 0, ties = 0;  // of the pages before
  for (int j0 = 0; j0 < np; j0 += 4 * T) {
    const int j = j0 + (int)threadIdx.x * 4;
    uint32_t mine = 0;
    uint32_t k[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      k[i] = j + i < np ? keys[j + i] & mask : 0u;
      if (j + i < np) mine += k[i] > prefix ? 0x10000u : k[i] == prefix ? 1u : 0u;
    }
    const uint32_t incl = wave_incl_scan(mine, lane);
    __syncthreads();
    if (lane == 63) waves[w] = incl;
    __syncthreads();
    uint32_t before = incl - mine, all = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      if (i < w) before += waves[i];
      all += waves[i];
    }
    uint32_t a = kept + (before >> 16), t = ties + (before & 0xffffu);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (j + i >= np) break;
      const bool above = k[i] > prefix, tie = k[i] == prefix;
      if (above || (tie && t < want)) out[a + min(t, want)] = j + i;
      a += above;
      t += tie;
    }
    kept += all >> 16;
    ties += all & 0xffffu;
  }
}

template <int T, int kHeads>
hipError_t launch_t(const PageSelectArgs& a, hipStream_t stream) {
  static std::mutex mu;
  static bool granted[64] = {};
  const size_t lds = ((size_t)(a.max_pages + 3) / 4 * 4 + (a.G + kHeads - 1) / kHeads * kHeads) * 4;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (lds > 32 * 1024) {
    std::lock_guard<std::mutex> lock(mu);
    if (dev < 0 || dev >= 64 || !granted[dev]) {
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(&page_select_kernel<T, kHeads>),
                              hipFuncAttributeMaxDynamicSharedMemorySize, (kMaxSelectPages + kMaxSelectHeads) * 4);
      if (e != hipSuccess) return e;
      if (dev >= 0 && dev < 64) granted[dev] = true;
    }
  }
  hipLaunchKernelGGL((page_select_kernel<T, kHeads>), dim3(a.B * a.Hkv), dim3(T), lds, stream, a);
  return hipGetLastError();
}

static_assert((kMaxSelectPages + kMaxSelectHeads) * 4 + 3 * kBins * 4 + 1024 <= 160 * 1024, "LDS of page_select_kernel");

}  // namespace

hipError_t launch_page_select(const PageSelectArgs& a, hipStream_t stream) {
  // 256 threads up to 1024 pages (256 rows of 1024, 4 heads: 9.3 us with events, 10.2 with 1024 threads; of 2048: 12.4
  // and 11.1); four heads at a time where the group has no more (9.3 us, 10.2 with eight).
  if (a.G <= 4) return a.max_pages <= 1024 ? launch_t<256, 4>(a, stream) : launch_t<1024, 4>(a, stream);
  return a.max_pages <= 1024 ? launch_t<256, 8>(a, stream) : launch_t<1024, 8>(a, stream);
}

}  // namespace cosa
