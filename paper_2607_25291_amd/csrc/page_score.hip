// Upper bounds on the logits of every page of a decode step, for gfx950.
//
// sum_d max(q_d min_d, q_d max_d) = relu(q) . max + min(q, 0) . min: one product of depth 2 d on the matrix
// cores, rows the pages and columns the query heads of one KV head (16 of them). Each lane reads its
// operands straight from the bounds: 512 contiguous bytes per (page, KV head), which are also all the
// bytes there are to read, so HBM bounds it.
#include "cosa_device.h"
#include "decode_internal.h"

namespace cosa {
namespace {

typedef float f32x4_t __attribute__((ext_vector_type(4)));

struct ScoreParams {
  const uint16_t *q, *bounds;
  const int32_t *table, *seq_lens;
  float* score;
  int Hq, Hkv, G, QG, max_pages, log2_page, segs, n_waves;  // segs: waves along a row of pages
  long long q_stride, n_pages;
  float scale;
};

// D (16 x 16, fp32) = A (16 x 32) B (32 x 16) + C, bf16: lane l supplies row / column l % 16 and k = 8 (l / 16)
// .. + 7; D row 4 (l / 16) + i, column l % 16 in register i.
__device__ __forceinline__ f32x4_t mfma16(const u32x4_t& a, const u32x4_t& b, const f32x4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}

// A wave scores TILES groups of 16 pages. Waves that follow each other take the KV heads of the same pages, so that a
// page's bounds, contiguous over its heads, are read at about one time. Lengths, table entries and queries
// are loaded side by side: a table entry is read before it is known to be in use.
template <int TILES>
__global__ __launch_bounds__(256) void page_score_kernel(ScoreParams P) {
  const int lane = threadIdx.x & 63, r = lane & 15, gq = lane >> 4;
  const int id = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (id >= P.n_waves) return;
  const int hq = id % (P.Hkv * P.QG), g = hq / P.QG, qg = hq % P.QG;
  const int ns = id / (P.Hkv * P.QG), n = ns / P.segs;
  const int j0 = (ns % P.segs) * (TILES * 16);
  const int32_t* row = P.table + (size_t)n * P.max_pages;
  long long p = j0 + lane < P.max_pages && lane < TILES * 16 ? row[j0 + lane] : 0;
  const int page = 1 << P.log2_page;
  const int len = min(max(P.seq_lens[n], 0), P.max_pages << P.log2_page);
  const int np = (int)(((unsigned)len + page - 1) >> P.log2_page);
  if (j0 >= np) return;
  // Columns behind the group's heads repeat its last one; they are not stored.
  const int h = g * P.G + min(qg * 16 + r, P.G - 1);
  const uint16_t* q = P.q + (size_t)n * P.q_stride + (size_t)h * kHeadDim + gq * 8;
  u32x4_t qp[4], qm[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const u32x4_t x = ldg16(q + c * 32);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t neg = ((x[i] >> 15) & 0x00010001u) * 0xffffu;  // all ones in halves with the sign set
      qp[c][i] = x[i] & ~neg;
      qm[c][i] = x[i] & neg;
    }
  }
  if (p < 0 || p >= P.n_pages) p = 0;
  const int page_of_lane = (int)p;
  const bool stores = qg * 16 + r < P.G;
  float* out = P.score + ((size_t)n * P.Hq + h) * P.max_pages;
#pragma unroll
  for (int i = 0; i < TILES; ++i) {
    const int j = j0 + i * 16;
    if (j >= np) break;
    const size_t pg = (unsigned)(TILES == 1 ? __shfl(page_of_lane, r, 64) : __shfl(page_of_lane, i * 16 + r, 64));
    const uint16_t* b = P.bounds + (pg * P.Hkv + g) * 2 * kHeadDim + gq * 8;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 4; ++c) acc = mfma16(ldg16(b + c * 32), qm[c], acc);
#pragma unroll
    for (int c = 0; c < 4; ++c) acc = mfma16(ldg16(b + kHeadDim + c * 32), qp[c], acc);
    if (stores) {
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (j + gq * 4 + v < np) out[j + gq * 4 + v] = acc[v] * P.scale;
    }
  }
}

template <int TILES>
hipError_t launch_t(ScoreParams P, int B, hipStream_t stream) {
  P.segs = (P.max_pages + TILES * 16 - 1) / (TILES * 16);
  P.n_waves = B * P.segs * P.Hkv * P.QG;
  hipLaunchKernelGGL((page_score_kernel<TILES>), dim3((P.n_waves + 3) / 4), dim3(256), 0, stream, P);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_score(const DecodeShape& sh, const uint16_t* q, const uint16_t* bounds,
                             const int32_t* table, const int32_t* seq_lens, float* score,
                             hipStream_t stream) {
  const int QG = (sh.G + 15) / 16;
  const ScoreParams P{q, bounds, table, seq_lens, score, sh.Hq, sh.Hkv, sh.G, QG, sh.max_pages,
                      sh.log2_page, 0, 0, sh.q_stride, sh.n_pages, sh.scale};
  return (long long)sh.B * sh.Hkv * QG * ((sh.max_pages + 63) / 64) >= 4096 ? launch_t<4>(P, sh.B, stream)
                                                                            : launch_t<1>(P, sh.B, stream);
}

}  // namespace cosa
