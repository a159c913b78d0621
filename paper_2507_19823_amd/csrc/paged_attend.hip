// Attention over the paged 8-bit cache.
#include "paged.h"

namespace hca {

struct AttendArgs {
  const uint16_t* q;
  int64_t q_stride;
  const int32_t *cu, *lens, *tables;
  const uint8_t* kv;
  const float* scale;
  const uint16_t* open;
  float sm;                  // sm_scale * log2(e): the softmax runs on powers of two
  int32_t total, max_q, causal;
  uint16_t* y;
  float* lse;
};

template <bool E4M3> __device__ __forceinline__ void code_to_float(uint32_t w, float* x) {
  if (E4M3) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int)(int8_t)(w >> (8 * i));
  }
}

// One workgroup per query row and head; its four waves take tiles of 16 tokens in turn and their partial results
// (running maximum, sum, weighted values) are joined in LDS.
template <int D, bool BF16, bool E4M3>
__global__ __launch_bounds__(256) void paged_attend_kernel(PagedView V, AttendArgs a) {
  constexpr int NH = D / 64;
  __shared__ float s_m[4], s_l[4], s_y[4][D];
  const int hq = blockIdx.y, h = hq / V.gqa, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int l16 = lane & 15, g = lane >> 4;
  int i;
  const int b = paged_find(V.n_seqs, blockIdx.x, &i, [&](int s) { int f; return paged_rows(a.cu, s, a.total, &f); });
  if (b >= V.n_seqs) return;
  int row0;
  const int m = paged_rows(a.cu, b, a.total, &row0);
  if (i >= a.max_q) return;
  int n = a.lens[b];
  n = n < 0 ? 0 : n > (V.max_pages << V.lp) ? V.max_pages << V.lp : n;
  const int sees = a.causal ? (n - m + i + 1 < 0 ? 0 : n - m + i + 1) : n;
  const uint16_t* qp = a.q + (int64_t)(row0 + i) * a.q_stride + (int64_t)hq * D;
  float q[NH][16];
#pragma unroll
  for (int x = 0; x < NH; ++x)
#pragma unroll
    for (int e = 0; e < 16; ++e) q[x][e] = elem_to_float<BF16>(qp[64 * x + 16 * g + e]);
  float top = -1e30f, sum = 0.f, y[NH][4];
#pragma unroll
  for (int x = 0; x < NH; ++x)
#pragma unroll
    for (int u = 0; u < 4; ++u) y[x][u] = 0.f;
  const int whole = n >> V.lp << V.lp;              // tokens from here on are open rows
  for (int t0 = w * 16; t0 < sees; t0 += 64) {
    float k[NH][16], v[NH][16], ks = 1.f, vs = 1.f;
    if (t0 < whole) {
      const int page = a.tables[(int64_t)b * V.max_pages + (t0 >> V.lp)];
      if (page < 0 || page >= V.n_pages) continue;
      const int64_t at = ((int64_t)page * V.hkv + h) * 2;
      const uint4* kp = reinterpret_cast<const uint4*>(a.kv + at * V.side() + (t0 & (V.P - 1)) * D);
      const uint4* vp = reinterpret_cast<const uint4*>(a.kv + (at + 1) * V.side() + (t0 & (V.P - 1)) * D);
      ks = a.scale[at];
      vs = a.scale[at + 1];
#pragma unroll
      for (int x = 0; x < NH; ++x) {
        const uint4 kw = kp[x * 64 + lane], vw = vp[x * 64 + lane];
        const uint32_t kk[4] = {kw.x, kw.y, kw.z, kw.w}, vv[4] = {vw.x, vw.y, vw.z, vw.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          code_to_float<E4M3>(kk[e], &k[x][4 * e]);
          code_to_float<E4M3>(vv[e], &v[x][4 * e]);
        }
      }
    } else {
      const uint16_t* kp = a.open + ((int64_t)b * V.hkv + h) * 2 * V.side() + (t0 & (V.P - 1)) * D;
      const uint16_t* vp = kp + V.side();
#pragma unroll
      for (int x = 0; x < NH; ++x)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          k[x][e] = elem_to_float<BF16>(kp[(x * 64 + lane) * 16 + e]);
          const bool live = t0 + 4 * g + (e & 3) < n;          // rows behind the last token may hold anything
          v[x][e] = live ? elem_to_float<BF16>(vp[(x * 64 + lane) * 16 + e]) : 0.f;
        }
    }
    float s = 0.f;
#pragma unroll
    for (int x = 0; x < NH; ++x)
#pragma unroll
      for (int e = 0; e < 16; ++e) s = fmaf(q[x][e], k[x][e], s);
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);                                      // token l16's score on every lane row
    s = t0 + l16 < sees ? s * (ks * a.sm) : -INFINITY;
    float mx = s;
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
    const float nt = fmaxf(top, mx), f = exp2f(top - nt);
    top = nt;
    float p = exp2f(s - nt);
    float ps = p;
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) ps += __shfl_xor(ps, d);
    sum = sum * f + ps;
    p *= vs;
    float pt[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) pt[j] = __shfl(p, 4 * g + j);
#pragma unroll
    for (int x = 0; x < NH; ++x)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        y[x][u] *= f;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[x][u] = fmaf(pt[j], v[x][4 * u + j], y[x][u]);
      }
  }
#pragma unroll
  for (int x = 0; x < NH; ++x)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      y[x][u] += __shfl_xor(y[x][u], 16);
      y[x][u] += __shfl_xor(y[x][u], 32);
      if (g == 0) s_y[w][64 * x + 16 * u + l16] = y[x][u];
    }
  if (lane == 0) { s_m[w] = top; s_l[w] = sum; }
  __syncthreads();
  const float all = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  float l = 0.f, out = 0.f;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const float f = exp2f(s_m[x] - all);
    l = fmaf(s_l[x], f, l);
    if (threadIdx.x < D) out = fmaf(s_y[x][threadIdx.x], f, out);
  }
  const int64_t o = (int64_t)(row0 + i) * V.hq + hq;
  if (threadIdx.x < D) a.y[o * D + threadIdx.x] = float_to_elem<BF16>(l > 0.f ? out / l : 0.f);
  if (threadIdx.x == 0 && a.lse != nullptr) a.lse[o] = l > 0.f ? (all + log2f(l)) * 0.693147180559945309f : -INFINITY;
}

template <int D, bool BF16>
static int32_t launch_attend_rows(const PagedView& V, const AttendArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)a.total, (unsigned)V.hq);
  if (V.code == HCA_E4M3)
    paged_attend_kernel<D, BF16, true><<<grid, 256, 0, st>>>(V, a);
  else
    paged_attend_kernel<D, BF16, false><<<grid, 256, 0, st>>>(V, a);
  HCA_HIP(hipGetLastError());
  return HCA_OK;
}

}  // namespace hca

using namespace hca;

extern "C" {

size_t hca_paged_workspace_bytes(const hca_paged_shape* shape, int64_t total_q, int32_t max_q) {
  PagedView V;
  if (paged_view(shape, &V) != HCA_OK || total_q < 0 || max_q < 0) return 0;
  return 256;
}

int32_t hca_paged_attend(const hca_paged_shape* shape, const void* q, int64_t q_stride, const int32_t* cu, int64_t total_q,
                         int32_t max_q, const int32_t* lens, int64_t max_len, const int32_t* tables, const void* kv,
                         const float* scale, const void* open, float sm_scale, int32_t causal, void* y, float* lse,
                         void* workspace, void* stream) {
  PagedView V;
  const int32_t rc = paged_view(shape, &V);
  if (rc != HCA_OK) return rc;
  if (cu == nullptr || lens == nullptr || tables == nullptr || kv == nullptr || scale == nullptr || open == nullptr ||
      workspace == nullptr || total_q < 0 || max_q < 0 || max_len < 0 || (total_q > 0 && (q == nullptr || y == nullptr)))
    return HCA_ERR_BAD_ARG;
  if (!(sm_scale > 0.0f)) return HCA_ERR_BAD_ARG;
  if (q_stride < (int64_t)V.hq * V.D || q_stride % 8 != 0) return HCA_ERR_BAD_ARG;
  if (!aligned16(q) || !aligned16(y) || !aligned16(kv) || !aligned16(open) || ((uintptr_t)workspace & 255) != 0) return HCA_ERR_BAD_ARG;
  if (total_q > (int64_t)1 << 26) return HCA_ERR_UNSUPPORTED;
  if (total_q == 0 || max_q == 0) return HCA_OK;
  const AttendArgs a{(const uint16_t*)q, q_stride, cu, lens, tables, (const uint8_t*)kv, scale, (const uint16_t*)open,
                     sm_scale * 1.44269504088896341f, (int32_t)total_q, max_q, causal, (uint16_t*)y, lse};
  hipStream_t st = (hipStream_t)stream;
  if (V.D == 128) return V.elem == HCA_BF16 ? launch_attend_rows<128, true>(V, a, st) : launch_attend_rows<128, false>(V, a, st);
  return V.elem == HCA_BF16 ? launch_attend_rows<64, true>(V, a, st) : launch_attend_rows<64, false>(V, a, st);
}

}  // extern "C"
