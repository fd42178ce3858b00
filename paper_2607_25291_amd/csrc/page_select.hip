// The pages that every KV head keeps of a decode step, for gfx950: one workgroup per (sequence, KV
// head).
//
// The rows' maxima, then one 32-bit key per page in LDS whose order is the order of selection (forced
// pages, NaN, then descending s). A radix selection over four 8-bit digits finds the K-th largest key and
// how many pages that equal it are kept; a scan over the pages then packs the kept ones in ascending
// order, so the list needs no sort.
#include <mutex>

#include "cosa_device.h"
#include "decode_internal.h"
#include "select_wave.h"

namespace cosa {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr uint32_t kForced = 0xffffffffu, kNan = 0xfffffffeu;

__device__ __forceinline__ uint32_t key_of(float s) {
  const uint32_t b = __float_as_uint(s + 0.f);  // -0 counts as 0
  if ((b & 0x7fffffffu) > 0x7f800000u) return kNan;
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

__global__ __launch_bounds__(kThreads) void page_select_kernel(PageSelectArgs A) {
  extern __shared__ uint32_t lds[];
  float* top = reinterpret_cast<float*>(lds);  // row maxima of the group's heads
  uint32_t* keys = lds + A.G;
  __shared__ uint32_t hist[256], waves[kWaves], pick[2];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int u = blockIdx.x, n = u / A.Hkv, g = u % A.Hkv;
  const int page = 1 << A.log2_page;
  const int len = min(max(A.seq_lens[n], 0), A.max_pages << A.log2_page);
  const int np = (int)(((unsigned)len + page - 1) >> A.log2_page);
  int32_t* out = A.pages + (size_t)u * A.max_keep;
  const int frac = (int)((A.fraction_micro * np + 999999) / 1000000);
  const int K = min(np, max(A.sink + A.recent, min(A.max_keep, max(A.min_keep, frac))));
  if (threadIdx.x == 0) A.count[u] = K;
  for (int j = K + threadIdx.x; j < A.max_keep; j += kThreads) out[j] = -1;
  if (K == np) {
    for (int j = threadIdx.x; j < K; j += kThreads) out[j] = j;
    return;
  }
  const float* score = A.score + ((size_t)n * A.Hq + (size_t)g * A.G) * A.max_pages;
  for (int h = w; h < A.G; h += kWaves) {
    float m = -INFINITY;
    for (int j = lane; j < np; j += 64) m = fmaxf(m, score[(size_t)h * A.max_pages + j]);
    m = wave_max(m);
    if (lane == 0) top[h] = m;
  }
  __syncthreads();
  for (int j = threadIdx.x; j < np; j += kThreads) {
    float s = -INFINITY;
    for (int h = 0; h < A.G; ++h) s = vmax(s, score[(size_t)h * A.max_pages + j] - top[h]);
    keys[j] = j < A.sink || j >= np - A.recent ? kForced : key_of(s);
  }

  uint32_t prefix = 0, mask = 0, want = (uint32_t)K;
  for (int shift = 24; shift >= 0; shift -= 8) {
    hist[threadIdx.x] = 0;
    __syncthreads();
    for (int j = threadIdx.x; j < np; j += kThreads)
      if ((keys[j] & mask) == prefix) atomicAdd(&hist[(keys[j] >> shift) & 255u], 1u);
    __syncthreads();
    if (w == 0) {
      // lane l holds bins 255 - 4 l .. 252 - 4 l: from the largest digit down
      uint32_t c[4], s = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) s += c[i] = hist[255 - 4 * lane - i];
      const uint32_t incl = wave_incl_scan(s, lane);
      uint32_t before = incl - s;
      if (before < want && incl >= want) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < want && before + c[i] >= want) {
            pick[0] = 255u - 4u * lane - i;
            pick[1] = want - before;
          }
          before += c[i];
        }
      }
    }
    __syncthreads();
    prefix |= pick[0] << shift;
    mask |= 255u << shift;
    want = pick[1];
  }

  // prefix is the K-th largest key; the first `want` pages that equal it are kept.
  uint32_t kept = 0, ties = 0;  // of the pages before
  for (int j0 = 0; j0 < np; j0 += kThreads) {
    const int j = j0 + threadIdx.x;
    const uint32_t key = j < np ? keys[j] : 0u;
    const bool above = j < np && key > prefix, tie = j < np && key == prefix;
    const uint64_t ba = __ballot(above), bt = __ballot(tie);
    __syncthreads();
    if (lane == 0) waves[w] = ((uint32_t)__popcll(ba) << 16) | (uint32_t)__popcll(bt);
    __syncthreads();
    uint32_t a = kept, t = ties;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      if (i < w) {
        a += waves[i] >> 16;
        t += waves[i] & 0xffffu;
      }
      kept += waves[i] >> 16;
      ties += waves[i] & 0xffffu;
    }
    a += lanes_below(ba);
    t += lanes_below(bt);
    if (above || (tie && t < want)) out[a + min(t, want)] = j;
  }
}

}  // namespace

hipError_t launch_page_select(const PageSelectArgs& a, hipStream_t stream) {
  static std::mutex mu;
  static bool granted[64] = {};
  const size_t lds = ((size_t)a.G + a.max_pages) * 4;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (lds > 60 * 1024) {
    std::lock_guard<std::mutex> lock(mu);
    if (dev < 0 || dev >= 64 || !granted[dev]) {
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(&page_select_kernel),
                              hipFuncAttributeMaxDynamicSharedMemorySize, 156 * 1024);
      if (e != hipSuccess) return e;
      if (dev >= 0 && dev < 64) granted[dev] = true;
    }
  }
  hipLaunchKernelGGL(page_select_kernel, dim3(a.B * a.Hkv), dim3(kThreads), lds, stream, a);
  return hipGetLastError();
}

}  // namespace cosa
