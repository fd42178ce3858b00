// Upper bounds on the logits of every page of a decode step, for gfx950.
//
// sum_d max(q_d min_d, q_d max_d) = relu(q) . max + min(q, 0) . min: one product of depth 2 d on the matrix
// cores, rows the pages and columns the query heads of one KV head (16 of them). Each lane reads its
// operands straight from the bounds: 512 contiguous bytes per (page, KV head), which are also all the
// bytes there are to read, so HBM bounds it.
#include "decode_device.h"
#include "decode_internal.h"

namespace cosa {
namespace {

struct ScoreParams {
  const uint16_t *q, *bounds;
  const int32_t *table, *seq_lens;
  float* score;
  int Hq, Hkv, G, QG, max_pages, log2_page, segs;  // segs: waves along a row of pages
  long long q_stride, n_pages;
  float scale;
  bool wide;  // rows of scores start on 16 bytes
};

// A wave scores 16 pages. Waves that follow each other take the KV heads of the same pages, so that a page's
// bounds, contiguous over its heads, are read at about one time. Lengths, table entries and queries are loaded
// side by side: a table entry is read before it is known to be in use. Bounds are read with loads that the caches do not
// keep: between two calls on a layer's bounds a step reads those of all other layers. Layers in turn with 1 / 32 / 64 / 128 /
// 489 MB of bounds each, 3 GB in all (64 MB with 1 MB): 3.1 / 8.6 / 15.4 / 26.3 / 104 us a call, with loads that are
// kept 2.9 / 9.1 / 16.5 / 29.4 / 105.
template <int NQ>
__global__ __launch_bounds__(64) void page_score_kernel(ScoreParams P) {
  const int lane = threadIdx.x, r = lane & 15, gq = lane >> 4;
  const int id = blockIdx.x;
  const int hq = id % (P.Hkv * P.QG), g = hq / P.QG, qg = hq % P.QG;
  const int ns = id / (P.Hkv * P.QG), n = ns / P.segs;
  const int j0 = (ns % P.segs) * kScorePages;
  const int32_t* row = P.table + (size_t)n * P.max_pages;
  long long p = j0 + r < P.max_pages ? row[j0 + r] : 0;
  const int page = 1 << P.log2_page;
  const int len = min(max(P.seq_lens[n], 0), P.max_pages << P.log2_page);
  const int np = (int)(((unsigned)len + page - 1) >> P.log2_page);
  if (j0 >= np) return;
  if (p < 0 || p >= P.n_pages) p = 0;
  const int page_of_lane = (int)p;
  u32x4_t qf[NQ][4];
  const uint16_t* q = P.q + (size_t)n * P.q_stride + gq * 8;
#pragma unroll
  for (int y = 0; y < NQ; ++y) {
    // Columns behind the group's heads repeat its last one; they are not stored.
    const int h = g * P.G + min((qg * NQ + y) * 16 + r, P.G - 1);
#pragma unroll
    for (int c = 0; c < 4; ++c) qf[y][c] = ldg16(q + (size_t)h * kHeadDim + c * 32);
  }
  RowOperands x;  // minimum, then maximum
  x.load(lane, [&](int k) __attribute__((always_inline)) {
    const size_t pg = (unsigned)__shfl(page_of_lane, k, 64);
    return P.bounds + (pg * P.Hkv + g) * 2 * kHeadDim;
  });
  x.to_operands();
#pragma unroll
  for (int y = 0; y < NQ; ++y) {
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      u32x4_t qp, qm;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t neg = ((qf[y][c][i] >> 15) & 0x00010001u) * 0xffffu;  // all ones in halves with the sign set
        qp[i] = qf[y][c][i] & ~neg;
        qm[i] = qf[y][c][i] & neg;
      }
      acc = mfma16(x.x[c], qm, acc);
      acc = mfma16(x.x[4 + c], qp, acc);
    }
    const int hh = (qg * NQ + y) * 16 + r;
    if (hh >= P.G) continue;
    float* out = P.score + ((size_t)n * P.Hq + g * P.G + hh) * P.max_pages + j0 + gq * 4;
    if (P.wide && j0 + gq * 4 + 3 < np) {
      *reinterpret_cast<f32x4_t*>(out) = acc * P.scale;
    } else {
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (j0 + gq * 4 + v < np) out[v] = acc[v] * P.scale;
    }
  }
}

}  // namespace

hipError_t launch_page_score(const DecodeShape& sh, const uint16_t* q, const uint16_t* bounds,
                             const int32_t* table, const int32_t* seq_lens, float* score,
                             hipStream_t stream) {
  const int QG = sh.G > 16 ? (sh.G + 31) / 32 : 1;  // a group's heads in 16 or 32 columns a wave
  const int segs = (sh.max_pages + kScorePages - 1) / kScorePages, n_waves = sh.B * segs * sh.Hkv * QG;
  const ScoreParams P{q, bounds, table, seq_lens, score, sh.Hq, sh.Hkv, sh.G, QG, sh.max_pages,
                      sh.log2_page, segs, sh.q_stride, sh.n_pages, sh.scale,
                      sh.max_pages % 4 == 0 && reinterpret_cast<uintptr_t>(score) % 16 == 0};
  if (sh.G > 16) hipLaunchKernelGGL((page_score_kernel<2>), dim3(n_waves), dim3(64), 0, stream, P);
  else hipLaunchKernelGGL((page_score_kernel<1>), dim3(n_waves), dim3(64), 0, stream, P);
  return hipGetLastError();
}

}  // namespace cosa
