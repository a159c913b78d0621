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


typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_raw(float x) { return __builtin_amdgcn_logf(x); }
__device__ __forceinline__ float lane_value(float v, int l) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), l)); }

// Four codes as four halves, exactly: an e4m3 number is a half, and so is an integer up to 127 (1024 + u in the
// mantissa's last bits, minus 1152, u = code + 128).
template <bool E4M3> __device__ __forceinline__ void code_to_half(uint32_t w, h2* x) {
  if (E4M3) {
    x[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
    x[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
  } else {
    const uint32_t u = w ^ 0x80808080u;
    const h2 off = {(_Float16)1152.f, (_Float16)1152.f};
    x[0] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - off;
    x[1] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - off;
  }
}
template <bool E4M3> __device__ __forceinline__ h8 codes_to_halves(uint32_t w0, uint32_t w1) {
  h2 x[4];
  code_to_half<E4M3>(w0, x);
  code_to_half<E4M3>(w1, x + 2);
  return h8{x[0].x, x[0].y, x[1].x, x[1].y, x[2].x, x[2].y, x[3].x, x[3].y};
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Maximum / sum over the four 16-lane rows of a wave, on every lane.
__device__ __forceinline__ float rows_max(float x) { return max_over_heads(x); }
__device__ __forceinline__ float rows_sum(float x) {
  const uint32_t xi = __float_as_uint(x);
  const auto r16 = __builtin_amdgcn_permlane16_swap(xi, xi, false, false);
  const float m = __uint_as_float(r16[0]) + __uint_as_float(r16[1]);
  const uint32_t mi = __float_as_uint(m);
  const auto r32 = __builtin_amdgcn_permlane32_swap(mi, mi, false, false);
  return __uint_as_float(r32[0]) + __uint_as_float(r32[1]);
}

// ---- few query rows: the cache is read once, at the rate of the memory ------------------------------
// All query rows of a sequence that share a KV head (queries x heads of the group, up to 16 NT of them) are the columns of one
// matrix product, so a token's codes are loaded and converted once.  Scores are computed transposed, S^T = K Q^T: then the
// lane that holds a column's scores is the lane that feeds them to Y^T = V^T P^T, and neither product needs data from
// another lane (the cache's order of values is the one in which S^T comes out).
//
// Everything is in halves on the matrix core: codes are halves exactly; a query row in bfloat16 is brought to halves with a
// power of two of its own (8 bits of mantissa fit in 11).  A page's key scale multiplies the score; its value scale goes into the
// exponent, w = 2^(x + log2 vs - M), so the running reference M bounds what the products see, whatever the scales.
// Weights are rounded to halves (2^-11 relative, the only rounding between the cache and the 32-bit sums; rounding at
// the output's own step) with M 12 below the running maximum: the halves then reach 2^-26 below it as normal numbers, 2^-36 in
// all, and M moves only when a score passes it by 15.  Their sum is taken in 32 bits before that, over w / vs.
//
// The tokens of a batch are divided evenly over the chip, from the lengths on the device: items of L units of 64
// tokens, L such that there are about as many items as fit at once.
constexpr int kUnit = 64;

struct SplitPlan {
  int32_t want;         // items per KV head, about: a sequence's last one may be short, so there are up to n_seqs more
  int32_t least;        // units per item at least
};
constexpr int kWholeSeq = 1 << 25;                     // as `least`: more units than a sequence can have

// tokens of sequence b, within the table
__device__ __forceinline__ int seq_len(const PagedView& V, const AttendArgs& a, int b) {
  const int n = a.lens[b], most = V.max_pages << V.lp;
  return n < 0 ? 0 : n > most ? most : n;
}
// units of whole pages of sequence b: at least one if it has queries
__device__ __forceinline__ int seq_units(const PagedView& V, const AttendArgs& a, int b) {
  int f;
  if (paged_rows(a.cu, b, a.total, &f) == 0) return 0;
  const int u = ((seq_len(V, a, b) >> V.lp << V.lp) + kUnit - 1) / kUnit;
  return u > 1 ? u : 1;
}
__device__ __forceinline__ int split_len(const PagedView& V, const AttendArgs& a, const SplitPlan& sp) {
  const int lane = threadIdx.x & 63;
  if (sp.least >= kWholeSeq) return kWholeSeq;
  uint64_t units = 0;
  for (int b = lane; b < V.n_seqs; b += 64) units += (uint64_t)seq_units(V, a, b);
  units = wave_scan_incl(units);
  const int64_t all = (int64_t)((uint64_t)wave_last((uint32_t)(units >> 32)) << 32 | wave_last((uint32_t)units));
  const int64_t L = (all + sp.want - 1) / sp.want;
  return (int)(L > sp.least ? L : sp.least);
}

struct Partial {          // of one item, KV head and row: reference, sum; the weighted values follow in another array
  float M, l;
};

template <int D, int NT, bool E4M3>
__global__ __launch_bounds__(256) void paged_rows_kernel(PagedView V, AttendArgs a, SplitPlan sp, Partial* __restrict__ ml,
                                                         float* __restrict__ part) {
  constexpr int NH = D / 64, NC = D / 16, COLS = 16 * NT;
  extern __shared__ float lds[];                       // [4][COLS][D + 4], then M and l of each wave [4][COLS]
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.y;
  const int L = split_len(V, a, sp);
  int it;
  const int b = paged_find(V.n_seqs, blockIdx.x, &it, [&](int s) { return (seq_units(V, a, s) + L - 1) / L; });
  if (b >= V.n_seqs) return;
  int row0;
  const int m_all = paged_rows(a.cu, b, a.total, &row0);
  const int m = m_all < a.max_q ? m_all : a.max_q;
  const int n = seq_len(V, a, b), G = V.gqa;
  const int whole = n >> V.lp << V.lp;
  const int units = seq_units(V, a, b);
  const int u0 = it * L, u1 = u0 + L < units ? u0 + L : units;
  const bool last = u1 == units;
  const int R = m * G;                                 // rows in use

  // this lane's query columns
  h8 q[NT][NH][2];
  float qs[NT];                                        // what a column's halves stand for, times sm_scale log2(e)
  int sees[NT], least_seen = n;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = 16 * nt + l16;
    const bool live = r < R;
    const int qi = live ? r / G : 0, hq = h * G + (live ? r % G : 0);
    const uint16_t* qp = a.q + (int64_t)(row0 + qi) * a.q_stride + (int64_t)hq * D;
    const int upto = n - m_all + qi + 1;
    sees[nt] = !(live && a.causal) ? n : upto > 0 ? upto : 0;
    if (sees[nt] < least_seen) least_seen = sees[nt];
    uint4 raw[NH][2];
#pragma unroll
    for (int x = 0; x < NH; ++x)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        raw[x][e] = live ? *reinterpret_cast<const uint4*>(qp + 64 * x + 16 * g + 8 * e) : uint4{0, 0, 0, 0};
    qs[nt] = a.sm;
    if (V.elem == HCA_BF16) {
      float amax = 0.f;
#pragma unroll
      for (int x = 0; x < NH; ++x)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            amax = fmaxf(amax, fmaxf(fabsf(elem_to_float<true>(word(raw[x][e], i) & 0xffffu)), fabsf(elem_to_float<true>(word(raw[x][e], i) >> 16))));
      amax = rows_max(amax);
      int ex = amax > 0.f ? 14 - ilogbf(amax) : 0;
      ex = ex > 100 ? 100 : ex;                        // largest magnitude in [2^14, 2^15)
      const float up = ldexpf(1.0f, ex);
      qs[nt] = ldexpf(a.sm, -ex);
#pragma unroll
      for (int x = 0; x < NH; ++x)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            q[nt][x][e][2 * i] = (_Float16)(elem_to_float<true>(word(raw[x][e], i) & 0xffffu) * up);
            q[nt][x][e][2 * i + 1] = (_Float16)(elem_to_float<true>(word(raw[x][e], i) >> 16) * up);
          }
    } else {
#pragma unroll
      for (int x = 0; x < NH; ++x)
#pragma unroll
        for (int e = 0; e < 2; ++e) q[nt][x][e] = __builtin_bit_cast(h8, raw[x][e]);
    }
  }
  least_seen = (int)wave_min((uint32_t)least_seen);

  float M[NT], l[NT];
  f4 y[NT][NC];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    M[nt] = -1e30f;
    l[nt] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) y[nt][c] = f4{0.f, 0.f, 0.f, 0.f};
  }

  // TT tiles of 16 tokens from t0 on: scores -> weights (halves, ready for the second product)
  const auto weigh = [&](auto tiles, f4(&s)[NT][decltype(tiles)::value], const float* ks, const float* lv, const float* iv, int t0,
                         int end, h2(&p)[NT][decltype(tiles)::value][2]) {
    constexpr int TT = decltype(tiles)::value;
    const bool masked = t0 + 16 * TT > (least_seen < end ? least_seen : end);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float d[TT][4];
      const int lim = sees[nt] < end ? sees[nt] : end;
      const auto scores = [&](float ref) {
#pragma unroll
        for (int tt = 0; tt < TT; ++tt) {
          const float c = ks[tt] * qs[nt], o = lv[tt] - ref;
#pragma unroll
          for (int i = 0; i < 4; ++i) d[tt][i] = fmaf(s[nt][tt][i], c, o);
        }
        if (masked) {
#pragma unroll
          for (int tt = 0; tt < TT; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (t0 + 16 * tt + 4 * g + i >= lim) d[tt][i] = -INFINITY;
        }
        float mx = d[0][0];
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i) mx = fmaxf(mx, d[tt][i]);
        return mx;
      };
      if (__any(scores(M[nt]) > 15.f)) {
        const float top = rows_max(scores(0.f)) - 12.f;
        const float next = fmaxf(M[nt], top), f = exp2_raw(M[nt] - next);
        M[nt] = next;
        l[nt] *= f;
#pragma unroll
        for (int c = 0; c < NC; ++c) y[nt][c] *= f;
        (void)scores(next);
      }
#pragma unroll
      for (int tt = 0; tt < TT; ++tt) {
        float e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = exp2_raw(d[tt][i]);
        l[nt] = fmaf((e[0] + e[1]) + (e[2] + e[3]), iv[tt], l[nt]);
        p[nt][tt][0] = h2{(_Float16)e[0], (_Float16)e[1]};
        p[nt][tt][1] = h2{(_Float16)e[2], (_Float16)e[3]};
      }
    }
  };

  // ---- whole pages: units u0 + w, u0 + w + 4, ...
  const int lpe = V.lp < 6 ? V.lp : 6;                  // pages smaller than a unit: 64 >> lpe of them per unit
  const int per = 64 >> lpe, group = 64 / per;          // pages per unit, units whose pages the lanes hold
  const int nk = u1 - u0 > w ? (u1 - u0 - w + 3) / 4 : 0;
  const int32_t* table = a.tables + (int64_t)b * V.max_pages;
  const int64_t side = V.side();
  // lane j holds page j % per of the wave's unit k0 + j / per: number (-1: no tokens), scales
  struct Info { int id; float ks, vs; };
  const auto fetch = [&](int k0) {
    const int k = k0 + lane / per, t = (u0 + w + 4 * k) * kUnit + (lane % per << lpe);
    Info f{-1, 0.f, 1.f};
    if (k < nk && t < whole) {
      const int id = table[t >> V.lp];
      if (id >= 0 && id < V.n_pages) {
        const float2 sc = *reinterpret_cast<const float2*>(a.scale + ((int64_t)id * V.hkv + h) * 2);
        f = Info{id, sc.x, sc.y};
      }
    }
    return f;
  };
  Info cur = fetch(0);
  float cur_lv = log2_raw(cur.vs), cur_iv = 1.0f / cur.vs;
  uint4 kw[4][NH], vw[4][NH];
  const auto address = [&](int k, int tt) {             // first key byte of tile tt of unit k; null: no tokens
    const int id = __builtin_amdgcn_readlane(cur.id, (k % group) * per + (16 * tt >> lpe));
    const int t = (u0 + w + 4 * k) * kUnit + 16 * tt;
    return id < 0 ? (const uint8_t*)nullptr : a.kv + ((int64_t)id * V.hkv + h) * 2 * side + (t & (V.P - 1)) * D;
  };
  const auto load = [&](int k, uint4(&x)[4][NH], int64_t off) {
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
      const uint8_t* p = address(k, tt);
#pragma unroll
      for (int z = 0; z < NH; ++z)
        x[tt][z] = p != nullptr ? load_stream16(reinterpret_cast<const uint4*>(p + off) + z * 64 + lane) : uint4{0, 0, 0, 0};
    }
  };
  if (nk > 0) {
    load(0, kw, 0);
    load(0, vw, side);
  }
  for (int k = 0; k < nk; ++k) {
    float ks[4], lv[4], iv[4];
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
      const int j = (k % group) * per + (16 * tt >> lpe);
      const bool none = __builtin_amdgcn_readlane(cur.id, j) < 0;
      ks[tt] = lane_value(cur.ks, j);
      lv[tt] = none ? -INFINITY : lane_value(cur_lv, j);
      iv[tt] = none ? 0.f : lane_value(cur_iv, j);
    }
    f4 s[NT][4];
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[nt][tt] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < NH; ++x)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const h8 kk = codes_to_halves<E4M3>(word(kw[tt][x], 2 * e), word(kw[tt][x], 2 * e + 1));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) s[nt][tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kk, q[nt][x][e], s[nt][tt], 0, 0, 0);
        }
    }
    const bool more = k + 1 < nk;
    if (more) {
      if ((k + 1) % group == 0) {
        cur = fetch(k + 1);
        cur_lv = log2_raw(cur.vs);
        cur_iv = 1.0f / cur.vs;
      }
      load(k + 1, kw, 0);
    }
    h2 p[NT][4][2];
    weigh(std::integral_constant<int, 4>{}, s, ks, lv, iv, (u0 + w + 4 * k) * kUnit, whole, p);
#pragma unroll
    for (int pr = 0; pr < 2; ++pr) {
      h8 pb[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
        pb[nt] = h8{p[nt][2 * pr][0].x, p[nt][2 * pr][0].y, p[nt][2 * pr][1].x, p[nt][2 * pr][1].y,
                    p[nt][2 * pr + 1][0].x, p[nt][2 * pr + 1][0].y, p[nt][2 * pr + 1][1].x, p[nt][2 * pr + 1][1].y};
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const h8 vv = codes_to_halves<E4M3>(word(vw[2 * pr][c >> 2], c & 3), word(vw[2 * pr + 1][c >> 2], c & 3));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) y[nt][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vv, pb[nt], y[nt][c], 0, 0, 0);
      }
    }
    if (more) load(k + 1, vw, side);
  }

  // ---- open rows, two tiles per wave, in the last item: the same with halves made from the rows themselves
  if (last) {
    const int t0 = whole + 32 * w;
    const auto widen = [&](uint32_t bits) { return V.elem == HCA_BF16 ? elem_to_float<true>(bits) : elem_to_float<false>(bits); };
    if (t0 < n) {
      const uint16_t* kp = a.open + ((int64_t)b * V.hkv + h) * 2 * side + (t0 & (V.P - 1)) * D;
      const bool two = t0 + 16 < n;                     // (a page of 16 has no second tile)
      h8 kk[2][NH][2], vv[2][NH][2];
      float ks[2], lv[2], iv[2];
#pragma unroll
      for (int sd = 0; sd < 2; ++sd) {
        uint4 raw[2][NH][2];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int x = 0; x < NH; ++x)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              uint4 v = uint4{0, 0, 0, 0};
              if (tt == 0 || two) v = *(reinterpret_cast<const uint4*>(kp + sd * side + tt * 16 * D + (x * 64 + lane) * 16) + e);
              // rows behind the last token may hold anything: keys by lane, values by place in the tile
              const int t = t0 + 16 * tt;
              uint32_t wd[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int a0 = sd == 0 ? t + l16 : t + 4 * g + 2 * (i & 1), a1 = sd == 0 ? t + l16 : a0 + 1;
                wd[i] = (a0 < n ? wd[i] & 0xffffu : 0u) | (a1 < n ? wd[i] & 0xffff0000u : 0u);
              }
              raw[tt][x][e] = uint4{wd[0], wd[1], wd[2], wd[3]};
            }
        // a power of two brings them to the halves' range: bfloat16 keys to the top of it (below it nothing is lost that
        // counts), values to that of codes, so that their weights are no smaller than a whole page's
        int ex = 0;
        if (sd == 1 || V.elem == HCA_BF16) {
          float amax = 0.f;
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int x = 0; x < NH; ++x)
#pragma unroll
              for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const uint32_t u = word(raw[tt][x][e], i);
                  amax = fmaxf(amax, fmaxf(fabsf(widen(u & 0xffffu)), fabsf(widen(u >> 16))));
                }
          amax = wave_max(amax);
          ex = amax > 0.f ? (sd == 0 ? 14 : 6) - ilogbf(amax) : 0;
          ex = ex > 64 ? 64 : ex;
        }
        const float up = ldexpf(1.0f, ex);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int x = 0; x < NH; ++x)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              h8 o = __builtin_bit_cast(h8, raw[tt][x][e]);
              if (sd == 1 || V.elem == HCA_BF16) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const uint32_t u = word(raw[tt][x][e], i);
                  o[2 * i] = (_Float16)(widen(u & 0xffffu) * up);
                  o[2 * i + 1] = (_Float16)(widen(u >> 16) * up);
                }
              }
              (sd == 0 ? kk : vv)[tt][x][e] = o;
            }
        if (sd == 0) ks[0] = ks[1] = ldexpf(1.0f, -ex);
        else {
          lv[0] = lv[1] = (float)-ex;
          iv[0] = iv[1] = up;
        }
      }
      f4 s[NT][2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          s[nt][tt] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int x = 0; x < NH; ++x)
#pragma unroll
            for (int e = 0; e < 2; ++e) s[nt][tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kk[tt][x][e], q[nt][x][e], s[nt][tt], 0, 0, 0);
        }
      h2 p[NT][2][2];
      weigh(std::integral_constant<int, 2>{}, s, ks, lv, iv, t0, n, p);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const h8 pb = h8{p[nt][0][0].x, p[nt][0][0].y, p[nt][0][1].x, p[nt][0][1].y,
                         p[nt][1][0].x, p[nt][1][0].y, p[nt][1][1].x, p[nt][1][1].y};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          // channels 16 c + l16: numbers 4 (c % 4) .. + 3 of the lane's sixteen
          const h8 v0 = vv[0][c >> 2][(c & 3) >> 1], v1 = vv[1][c >> 2][(c & 3) >> 1];
          const int o = 4 * (c & 1);
          y[nt][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
              h8{v0[o], v0[o + 1], v0[o + 2], v0[o + 3], v1[o], v1[o + 1], v1[o + 2], v1[o + 3]}, pb, y[nt][c], 0, 0, 0);
        }
      }
    }
  }

  // ---- the four waves' results are joined
  constexpr int RS = D + 4;
  float* sM = lds + 4 * COLS * RS;
  float* sl = sM + 4 * COLS;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float sum = rows_sum(l[nt]);
    if (g == 0) {
      sM[w * COLS + 16 * nt + l16] = M[nt];
      sl[w * COLS + 16 * nt + l16] = sum;
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
      *reinterpret_cast<f4*>(lds + (w * COLS + 16 * nt + l16) * RS + 16 * c + 4 * g) = y[nt][c];
  }
  __syncthreads();
  const bool only = units <= L;
  constexpr int TPR = D / 4;                            // threads per row, four channels each
  for (int r = threadIdx.x / TPR; r < R; r += 256 / TPR) {
    const int ch = threadIdx.x % TPR * 4;
    const float all = fmaxf(fmaxf(sM[r], sM[COLS + r]), fmaxf(sM[2 * COLS + r], sM[3 * COLS + r]));
    float sum = 0.f;
    f4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float f = exp2_raw(sM[x * COLS + r] - all);
      sum = fmaf(sl[x * COLS + r], f, sum);
      o += *reinterpret_cast<const f4*>(lds + (x * COLS + r) * RS + ch) * f;
    }
    if (only) {
      const int64_t at = (int64_t)(row0 + r / G) * V.hq + h * G + r % G;
      const float inv = sum > 0.f ? 1.0f / sum : 0.f;
      uint16_t u[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = V.elem == HCA_BF16 ? float_to_elem<true>(o[i] * inv) : float_to_elem<false>(o[i] * inv);
      *reinterpret_cast<uint2*>(a.y + at * D + ch) = uint2{u[0] | (uint32_t)u[1] << 16, u[2] | (uint32_t)u[3] << 16};
      if (ch == 0 && a.lse != nullptr) a.lse[at] = sum > 0.f ? (all + log2f(sum)) * 0.693147180559945309f : -INFINITY;
    } else {
      const int64_t at = ((int64_t)blockIdx.x * V.hkv + h) * COLS + r;
      *reinterpret_cast<f4*>(part + at * D + ch) = o;
      if (ch == 0) ml[at] = Partial{all, sum};
    }
  }
}

// Joins the items of sequences that have several.  One workgroup per query row and head, items in a fixed order.
template <int D>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedView V, AttendArgs a, SplitPlan sp, int cols, const Partial* __restrict__ ml,
                                                         const float* __restrict__ part) {
  constexpr int TPR = D / 4, NG = 256 / TPR;            // groups of threads, each with every NG-th item
  __shared__ f4 s_o[NG][TPR];
  __shared__ float s_l[NG];
  const int hq = blockIdx.y, h = hq / V.gqa, lane = threadIdx.x & 63;
  int i;
  const int b = paged_find(V.n_seqs, blockIdx.x, &i, [&](int s) { int f; return paged_rows(a.cu, s, a.total, &f); });
  if (b >= V.n_seqs || i >= a.max_q) return;
  const int L = split_len(V, a, sp);
  const int count = (seq_units(V, a, b) + L - 1) / L;
  if (count <= 1) return;
  uint32_t before = 0;
  for (int s = lane; s < b; s += 64) before += (uint32_t)((seq_units(V, a, s) + L - 1) / L);
  const int first = (int)wave_sum(before);
  int row0;
  (void)paged_rows(a.cu, b, a.total, &row0);
  const int r = i * V.gqa + hq % V.gqa;
  const int grp = threadIdx.x / TPR, ch = threadIdx.x % TPR * 4;
  const auto at = [&](int k) { return ((int64_t)(first + k) * V.hkv + h) * cols + r; };
  float M = -1e30f;
  for (int k = lane; k < count; k += 64) M = fmaxf(M, ml[at(k)].M);
  M = wave_max(M);
  float sum = 0.f;
  f4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int k = grp; k < count; k += NG) {
    const Partial p = ml[at(k)];
    const float f = exp2_raw(p.M - M);
    sum = fmaf(p.l, f, sum);
    o += *reinterpret_cast<const f4*>(part + at(k) * D + ch) * f;
  }
  s_o[grp][ch / 4] = o;
  if (ch == 0) s_l[grp] = sum;
  __syncthreads();
  if (grp != 0) return;
#pragma unroll
  for (int x = 1; x < NG; ++x) {
    o += s_o[x][ch / 4];
    sum += s_l[x];
  }
  const int64_t out = (int64_t)(row0 + i) * V.hq + hq;
  const float inv = sum > 0.f ? 1.0f / sum : 0.f;
  uint16_t u[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) u[x] = V.elem == HCA_BF16 ? float_to_elem<true>(o[x] * inv) : float_to_elem<false>(o[x] * inv);
  *reinterpret_cast<uint2*>(a.y + out * D + ch) = uint2{u[0] | (uint32_t)u[1] << 16, u[2] | (uint32_t)u[3] << 16};
  if (ch == 0 && a.lse != nullptr) a.lse[out] = sum > 0.f ? (M + log2f(sum)) * 0.693147180559945309f : -INFINITY;
}

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

// Items per KV head that fill the chip once: two workgroups on each of its 256 compute units.
static int rows_want(const PagedView& V) { return V.hkv >= 512 ? 1 : 512 / V.hkv; }
constexpr int kOneItem = 1024;      // sequences up to this length are one item, and nothing has to be joined

static int64_t rows_items(const PagedView& V, int64_t total_q) { return rows_want(V) + (total_q < V.n_seqs ? total_q : V.n_seqs); }
static int rows_cols(const PagedView& V, int max_q) {
  const int64_t R = (int64_t)max_q * V.gqa;
  return R <= 16 ? 16 : R <= 32 ? 32 : 64;
}

template <int D, int NT>
static int32_t launch_rows_nt(const PagedView& V, const AttendArgs& a, int64_t max_len, void* ws, hipStream_t st) {
  constexpr int lds = 4 * 16 * NT * (D + 4 + 2) * 4;
  const bool one = max_len <= kOneItem;
  const int64_t items = one ? V.n_seqs : rows_items(V, a.total);
  const SplitPlan sp{rows_want(V), one ? kWholeSeq : 4};
  Partial* ml = (Partial*)ws;
  float* part = (float*)((char*)ws + align_up(items * V.hkv * 16 * NT * (int64_t)sizeof(Partial), 256));
  const dim3 grid((unsigned)items, (unsigned)V.hkv);
  const auto kernel = V.code == HCA_E4M3 ? paged_rows_kernel<D, NT, true> : paged_rows_kernel<D, NT, false>;
  if (lds > 65536) {
    static std::atomic<uint64_t> done[2];
    const int32_t rc = lds_opt_in((const void*)kernel, lds, &done[V.code == HCA_E4M3]);
    if (rc != HCA_OK) return rc;
  }
  kernel<<<grid, 256, lds, st>>>(V, a, sp, ml, part);
  HCA_HIP(hipGetLastError());
  if (!one) {
    paged_join_kernel<D><<<dim3((unsigned)a.total, (unsigned)V.hq), 256, 0, st>>>(V, a, sp, 16 * NT, ml, part);
    HCA_HIP(hipGetLastError());
  }
  return HCA_OK;
}
template <int D>
static int32_t launch_rows(const PagedView& V, const AttendArgs& a, int64_t max_len, void* ws, hipStream_t st) {
  switch (rows_cols(V, a.max_q)) {
    case 16: return launch_rows_nt<D, 1>(V, a, max_len, ws, st);
    case 32: return launch_rows_nt<D, 2>(V, a, max_len, ws, st);
    default: return launch_rows_nt<D, 4>(V, a, max_len, ws, st);
  }
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
  if (max_q > total_q) max_q = (int32_t)total_q;
  const int64_t rows = rows_items(V, total_q) * V.hkv * rows_cols(V, max_q);
  return (size_t)(align_up(rows * (int64_t)sizeof(Partial), 256) + align_up(rows * V.D * 4, 256) + 256);
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
                     sm_scale * 1.44269504088896341f, (int32_t)total_q, (int32_t)(max_q < total_q ? max_q : total_q), causal, (uint16_t*)y, lse};
  hipStream_t st = (hipStream_t)stream;
  if ((int64_t)(max_q < total_q ? max_q : total_q) * V.gqa <= 64)
    return V.D == 128 ? launch_rows<128>(V, a, max_len, workspace, st) : launch_rows<64>(V, a, max_len, workspace, st);
  if (V.D == 128) return V.elem == HCA_BF16 ? launch_attend_rows<128, true>(V, a, st) : launch_attend_rows<128, false>(V, a, st);
  return V.elem == HCA_BF16 ? launch_attend_rows<64, true>(V, a, st) : launch_attend_rows<64, false>(V, a, st);
}

}  // extern "C"
