// Paged 8-bit cache: page tables and slot maps, and the store that codes whole blocks.
#include "paged.h"

namespace hca {

int32_t paged_view(const hca_paged_shape* s, PagedView* V) {
  if (s == nullptr) return HCA_ERR_BAD_ARG;
  if (s->n_seqs < 1 || s->n_q_heads < 1 || s->n_kv_heads < 1 || s->max_pages < 1 || s->n_pages < 1) return HCA_ERR_BAD_ARG;
  if (s->n_q_heads % s->n_kv_heads != 0) return HCA_ERR_BAD_ARG;
  if (s->n_seqs > kPagedMaxSeqs || s->n_kv_heads > 1024 || s->n_q_heads / s->n_kv_heads > kPagedMaxGqa) return HCA_ERR_UNSUPPORTED;
  if (!(s->head_dim == 64 || s->head_dim == 128)) return HCA_ERR_UNSUPPORTED;
  if (!(s->page == 16 || s->page == 32 || s->page == 64 || s->page == 128)) return HCA_ERR_UNSUPPORTED;
  if (!(s->elem == HCA_F16 || s->elem == HCA_BF16) || !(s->code == HCA_INT8 || s->code == HCA_E4M3)) return HCA_ERR_UNSUPPORTED;
  if ((int64_t)s->max_pages * s->page > (int64_t)1 << 30) return HCA_ERR_UNSUPPORTED;
  if ((int64_t)s->n_seqs * s->max_pages > ((int64_t)1 << 37) / s->page) return HCA_ERR_UNSUPPORTED;   // tokens of all rows
  if (s->n_pages > INT32_MAX / s->page) return HCA_ERR_UNSUPPORTED;   // slots are int32
  V->n_seqs = s->n_seqs;
  V->hq = s->n_q_heads;
  V->hkv = s->n_kv_heads;
  V->gqa = s->n_q_heads / s->n_kv_heads;
  V->D = s->head_dim;
  V->P = s->page;
  V->lp = __builtin_ctz((unsigned)s->page);
  V->max_pages = s->max_pages;
  V->elem = s->elem;
  V->code = s->code;
  V->n_pages = s->n_pages;
  return HCA_OK;
}

// ---- page tables -----------------------------------------------------------------------------------
// One workgroup, a thread per sequence: three prefix sums (tokens, pages given back, pages needed) and the pages
// moved by whole waves.  Nothing but latency: lengths, counts and the free list's top are a few KB.
struct MapArgs {
  const int32_t *add, *lens_in, *free_in;
  int32_t *lens_out, *tables, *free_pages, *free_out, *start, *cu, *tok_seq, *tok_pos, *tok_slot;
  int64_t max_new;
};

// Sequence, position and slot of new token t; c = the running sums (device or LDS), c[0] = 0.
__device__ __forceinline__ void map_token(const PagedView& V, const MapArgs& a, const int32_t* c, const int32_t* start, int t) {
  int lo = 0, hi = V.n_seqs - 1;                     // the last sequence whose first row is not behind t
  while (lo < hi) {
    const int m = (lo + hi + 1) >> 1;
    if (c[m] <= t) lo = m; else hi = m - 1;
  }
  const int s = start[lo];
  const int pos = s < 0 ? -1 : s + (t - c[lo]);
  if (a.tok_seq != nullptr) a.tok_seq[t] = lo;
  if (a.tok_pos != nullptr) a.tok_pos[t] = pos;
  if (a.tok_slot != nullptr)
    a.tok_slot[t] = pos < 0 ? -1 : a.tables[(int64_t)lo * V.max_pages + (pos >> V.lp)] * V.P + (pos & (V.P - 1));
}

constexpr int kMapThreads = 1024;

__global__ __launch_bounds__(kMapThreads) void paged_map_kernel(PagedView V, MapArgs a, int tokens_here) {
  __shared__ uint64_t wsum[16];
  __shared__ int32_t s_cu[kPagedMaxSeqs + 1], s_start[kPagedMaxSeqs];
  __shared__ int32_t s_first[kPagedMaxSeqs], s_count[kPagedMaxSeqs];      // table entries to move
  __shared__ int64_t s_rank[kPagedMaxSeqs];                               // places in the free list
  const int b = threadIdx.x, w = b >> 6, lane = b & 63;
  const bool live = b < V.n_seqs;
  const int64_t room = (int64_t)V.max_pages << V.lp;
  int64_t n = live ? a.lens_in[b] : 0;
  n = n < 0 ? 0 : n > room ? room : n;
  const int add = live ? a.add[b] : 0;
  int64_t fc = a.free_in[0];
  fc = fc < 0 ? 0 : fc > V.n_pages ? V.n_pages : fc;
  const bool gone = add < 0;
  const int64_t T = add > 0 ? add : 0;
  const int64_t held = (n + V.P - 1) >> V.lp;
  // pages of ending sequences go on top of the free list
  const auto scan = [&](int64_t x, int64_t* all) {
    uint64_t sum;
    const int64_t before = (int64_t)block_scan_excl<16>((uint64_t)x, wsum, &sum);
    *all = (int64_t)sum;
    return before;
  };
  int64_t back_all, need_all, T_all;
  const int64_t back = gone ? held : 0;
  const int64_t back_at = scan(back, &back_all);
  s_first[b] = 0;
  s_count[b] = (int32_t)back;
  s_rank[b] = fc + back_at;
  __syncthreads();
  for (int s = w; s < V.n_seqs; s += 16) {
    const int32_t* row = a.tables + (int64_t)s * V.max_pages;
    for (int j = lane; j < s_count[s]; j += 64)
      if (s_rank[s] + j < V.n_pages) a.free_pages[s_rank[s] + j] = row[j];
  }
  int64_t avail = fc + back_all;
  if (avail > V.n_pages) avail = V.n_pages;
  const int64_t n0 = gone ? 0 : n;
  const int64_t row0 = scan(T, &T_all);
  const bool fits = n0 + T <= room && row0 + T <= a.max_new;
  const int64_t first = (n0 + V.P - 1) >> V.lp;
  const int64_t need = fits ? ((n0 + T + V.P - 1) >> V.lp) - first : 0;
  const int64_t need_at = scan(need, &need_all);
  const bool ok = fits && (need == 0 || need_at + need <= avail);
  int64_t given;
  (void)scan(ok ? need : 0, &given);
  s_first[b] = (int32_t)first;
  s_count[b] = ok ? (int32_t)need : 0;
  s_rank[b] = avail - 1 - need_at;
  const int32_t st = ok ? (int32_t)n0 : -1;
  s_start[b] = st;
  s_cu[b] = (int32_t)(row0 < a.max_new ? row0 : a.max_new);
  if (b == 0) s_cu[V.n_seqs] = (int32_t)(T_all < a.max_new ? T_all : a.max_new);
  if (live) {
    a.start[b] = st;
    a.lens_out[b] = (int32_t)(n0 + (ok ? T : 0));
    a.cu[b] = s_cu[b];
    if (b == 0) {
      a.cu[V.n_seqs] = s_cu[V.n_seqs];
      a.free_out[0] = (int32_t)(avail - given);
    }
  }
  __syncthreads();           // the pushed pages are in place, and so are the lists
  for (int s = w; s < V.n_seqs; s += 16) {
    int32_t* row = a.tables + (int64_t)s * V.max_pages + s_first[s];
    for (int j = lane; j < s_count[s]; j += 64) row[j] = a.free_pages[s_rank[s] - j];
  }
  if (!tokens_here) return;
  __syncthreads();
  for (int t = b; t < s_cu[V.n_seqs]; t += kMapThreads) map_token(V, a, s_cu, s_start, t);
}

// the same for many tokens: a thread each, in a launch of its own
__global__ __launch_bounds__(256) void paged_slots_kernel(PagedView V, MapArgs a) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t < a.cu[V.n_seqs]) map_token(V, a, a.cu, a.start, (int)t);
}

// ---- store -----------------------------------------------------------------------------------------
// blocks of sequence b that become whole, or 1 if none does but there are new tokens
struct StoreArgs {
  const uint16_t* x[2];       // keys, values
  int64_t stride[2];
  int32_t total;
  const int32_t *start, *cu, *tables;
  uint8_t* kv;
  float* scale;
  uint16_t* open;
};

__device__ __forceinline__ int store_items(const PagedView& V, const StoreArgs& a, int b) {
  int row;
  const int T = paged_rows(a.cu, b, a.total, &row), s = a.start[b];
  if (T == 0 || s < 0) return 0;
  const int c = (int)((((int64_t)s + T) >> V.lp) - (s >> V.lp));
  return c > 1 ? c : 1;
}

// One workgroup per (block, KV head, side).  The block's rows are staged in LDS as they are (rows of D numbers, 8 bytes
// of padding: the value pieces gather four rows at a time), their largest magnitude is reduced, and every thread codes
// pieces of 16 numbers in the cache's order.  The workgroup of a sequence's first block also writes the rows that
// stay open behind the last whole block: it alone reads old open rows, so nothing is overwritten before it is read.
template <int D, bool BF16, bool E4M3>
__global__ __launch_bounds__(256) void paged_store_kernel(PagedView V, StoreArgs a) {
  constexpr int RS = D + 4;                     // row stride in LDS
  extern __shared__ uint16_t rows[];            // [P][RS]
  __shared__ float wmax[4];
  const int h = blockIdx.y, side = blockIdx.z, tid = threadIdx.x;
  int m;
  const int b = paged_find(V.n_seqs, blockIdx.x, &m, [&](int s) { return store_items(V, a, s); });
  if (b >= V.n_seqs) return;
  int row0;
  const int T = paged_rows(a.cu, b, a.total, &row0), start = a.start[b];
  const int P = V.P;
  const int64_t end = (int64_t)start + T;
  const int nb = (start >> V.lp) + m;           // the block
  const int whole = (int)((end >> V.lp) - (start >> V.lp));
  const uint16_t* src = a.x[side] + (int64_t)h * D;
  const int64_t stride = a.stride[side];
  uint16_t* open = a.open + (((int64_t)b * V.hkv + h) * 2 + side) * V.side();
  if (whole > 0) {
    const int64_t p0 = (int64_t)nb << V.lp;
    const int old = p0 < start ? (int)(start - p0) : 0;      // rows that are in the open rows
    for (int i = tid; i < P * (D / 4); i += 256) {           // 8 bytes at a time
      const int o = i / (D / 4), ch = i % (D / 4) * 4;
      uint2 v;
      if (o >= old) {
        v = *reinterpret_cast<const uint2*>(src + (row0 + (p0 + o - start)) * stride + ch);
      } else {
        uint32_t e[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) e[k] = open[side == 0 ? key_at(o, ch + k, D) : value_at(o, ch + k, D)];
        v = uint2{e[0] | e[1] << 16, e[2] | e[3] << 16};
      }
      *reinterpret_cast<uint2*>(rows + o * RS + ch) = v;
    }
    __syncthreads();
    float amax = 0.f;
    for (int i = tid; i < P * (D / 4); i += 256) {
      const uint2 v = *reinterpret_cast<const uint2*>(rows + i / (D / 4) * RS + i % (D / 4) * 4);
      amax = fmaxf(amax, fmaxf(fmaxf(fabsf(elem_to_float<BF16>(v.x & 0xffffu)), fabsf(elem_to_float<BF16>(v.x >> 16))),
                               fmaxf(fabsf(elem_to_float<BF16>(v.y & 0xffffu)), fabsf(elem_to_float<BF16>(v.y >> 16)))));
    }
    amax = wave_max(amax);
    if ((tid & 63) == 0) wmax[tid >> 6] = amax;
    __syncthreads();
    amax = fmaxf(fmaxf(wmax[0], wmax[1]), fmaxf(wmax[2], wmax[3]));
    constexpr float kMax = E4M3 ? 448.f : 127.f;
    float scale = amax / kMax;
    if (!(scale >= 0x1p-64f)) scale = 0x1p-64f;
    const float inv = 1.0f / scale;
    const int page = nb < V.max_pages ? a.tables[(int64_t)b * V.max_pages + nb] : -1;
    if (page >= 0 && page < V.n_pages) {
      uint8_t* out = a.kv + (((int64_t)page * V.hkv + h) * 2 + side) * V.side();
      if (tid == 0) a.scale[((int64_t)page * V.hkv + h) * 2 + side] = scale;
      for (int i = tid; i < P * D / 16; i += 256) {            // piece i: 16 codes
        const int tile = i / (D / 16 * 16), r = i % (D / 16 * 16), hh = r >> 6, g = (r >> 4) & 3, l = r & 15;
        uint32_t wd[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float x[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            // keys: token l, channel 64 hh + 16 g + 4 k + j; values: token 4 g + j, channel 64 hh + 16 k + l
            const int t = 16 * tile + (side == 0 ? l : 4 * g + j);
            const int ch = 64 * hh + (side == 0 ? 16 * g + 4 * k + j : 16 * k + l);
            const float y = elem_to_float<BF16>(rows[t * RS + ch]) * inv;
            x[j] = fminf(fmaxf(y, -kMax), kMax);
          }
          if (E4M3) {
            int p = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
            p = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], p, true);
            wd[k] = (uint32_t)p;
          } else {
            wd[k] = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) wd[k] |= ((uint32_t)(int)rintf(x[j]) & 255u) << (8 * j);
          }
        }
        reinterpret_cast<uint4*>(out)[i] = uint4{wd[0], wd[1], wd[2], wd[3]};
      }
    }
  }
  if (m != 0) return;
  // rows of the block that stays open (all new ones, if no block became whole)
  const int64_t first = whole > 0 ? end >> V.lp << V.lp : start;
  const int left = (int)(end - first);
  for (int i = tid; i < left * D; i += 256) {
    const int64_t p = first + i / D;
    const int o = (int)(p & (P - 1)), ch = i % D;
    open[side == 0 ? key_at(o, ch, D) : value_at(o, ch, D)] = src[(row0 + (p - start)) * stride + ch];
  }
}

template <int D, bool BF16>
static int32_t launch_store(const PagedView& V, const StoreArgs& a, dim3 grid, hipStream_t st) {
  const int lds = V.P * (D + 4) * 2;
  if (V.code == HCA_E4M3)
    paged_store_kernel<D, BF16, true><<<grid, 256, lds, st>>>(V, a);
  else
    paged_store_kernel<D, BF16, false><<<grid, 256, lds, st>>>(V, a);
  HCA_HIP(hipGetLastError());
  return HCA_OK;
}

}  // namespace hca

using namespace hca;

extern "C" {

size_t hca_paged_cache_bytes(const hca_paged_shape* shape) {
  PagedView V;
  return paged_view(shape, &V) == HCA_OK ? (size_t)(V.n_pages * V.page_bytes()) : 0;
}

size_t hca_paged_scale_bytes(const hca_paged_shape* shape) {
  PagedView V;
  return paged_view(shape, &V) == HCA_OK ? (size_t)V.n_pages * V.hkv * 2 * sizeof(float) : 0;
}

size_t hca_paged_open_bytes(const hca_paged_shape* shape) {
  PagedView V;
  return paged_view(shape, &V) == HCA_OK ? (size_t)V.n_seqs * V.page_bytes() * 2 : 0;
}

int32_t hca_paged_map(const hca_paged_shape* shape, const int32_t* add, const int32_t* lens_in, int32_t* lens_out,
                      int32_t* tables, int32_t* free_pages, const int32_t* free_in, int32_t* free_out, int64_t max_new,
                      int32_t* start, int32_t* cu, int32_t* tok_seq, int32_t* tok_pos, int32_t* tok_slot, void* stream) {
  PagedView V;
  const int32_t rc = paged_view(shape, &V);
  if (rc != HCA_OK) return rc;
  if (add == nullptr || lens_in == nullptr || lens_out == nullptr || tables == nullptr || free_pages == nullptr ||
      free_in == nullptr || free_out == nullptr || start == nullptr || cu == nullptr || max_new < 0)
    return HCA_ERR_BAD_ARG;
  if (max_new > (int64_t)1 << 30) return HCA_ERR_UNSUPPORTED;
  const MapArgs a{add, lens_in, free_in, lens_out, tables, free_pages, free_out, start, cu, tok_seq, tok_pos, tok_slot, max_new};
  const bool tokens = (tok_seq != nullptr || tok_pos != nullptr || tok_slot != nullptr) && max_new > 0;
  const bool here = tokens && max_new <= 2048;
  paged_map_kernel<<<1, kMapThreads, 0, (hipStream_t)stream>>>(V, a, here ? 1 : 0);
  HCA_HIP(hipGetLastError());
  if (tokens && !here) {
    paged_slots_kernel<<<(unsigned)((max_new + 255) / 256), 256, 0, (hipStream_t)stream>>>(V, a);
    HCA_HIP(hipGetLastError());
  }
  return HCA_OK;
}

int32_t hca_paged_store(const hca_paged_shape* shape, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                        int64_t total, const int32_t* start, const int32_t* cu, const int32_t* tables, void* kv,
                        float* scale, void* open, void* stream) {
  PagedView V;
  const int32_t rc = paged_view(shape, &V);
  if (rc != HCA_OK) return rc;
  if (start == nullptr || cu == nullptr || tables == nullptr || kv == nullptr || scale == nullptr || open == nullptr ||
      total < 0 || (total > 0 && (k == nullptr || v == nullptr)))
    return HCA_ERR_BAD_ARG;
  const int64_t least = (int64_t)V.hkv * V.D;
  if (k_stride < least || v_stride < least || k_stride % 8 != 0 || v_stride % 8 != 0) return HCA_ERR_BAD_ARG;
  if (!aligned16(k) || !aligned16(v) || !aligned16(kv) || !aligned16(open)) return HCA_ERR_BAD_ARG;
  if (total > (int64_t)1 << 30) return HCA_ERR_UNSUPPORTED;
  if (total == 0) return HCA_OK;
  const StoreArgs a{{(const uint16_t*)k, (const uint16_t*)v}, {k_stride, v_stride}, (int32_t)total, start, cu, tables,
                    (uint8_t*)kv, scale, (uint16_t*)open};
  // a sequence with T rows has at most (T + P - 1) / P <= T / P + 1 items
  const int64_t items = total / V.P + (total < V.n_seqs ? total : V.n_seqs);
  const dim3 grid((unsigned)items, (unsigned)V.hkv, 2);
  hipStream_t st = (hipStream_t)stream;
  if (V.D == 128) return V.elem == HCA_BF16 ? launch_store<128, true>(V, a, grid, st) : launch_store<128, false>(V, a, grid, st);
  return V.elem == HCA_BF16 ? launch_store<64, true>(V, a, grid, st) : launch_store<64, false>(V, a, grid, st);
}

}  // extern "C"
