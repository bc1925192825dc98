// Per-head RMSNorm of queries and keys and their rotation in one pass, its
// backward, and the append of a chunk's keys and values to the paged cache.
//
//   n = x rsqrt(mean x^2 + eps) g,   y_i = n_i cos a_i - n_{i+dh/2} sin a_i,
//   y_{i+dh/2} = n_{i+dh/2} cos a_i + n_i sin a_i,   a_i = pos[axis(i)] base^(-2i/dh)
//
// Bound by HBM: every head vector is read and written once.  A lane holds 8
// dimensions of the first half of a head and the matching 8 of the second (16-byte
// accesses, the pairs of a rotation in one lane), dh / 16 lanes a head, so a wave
// takes 1024 / dh heads of a row at a time.  The row's dh / 2 angles are formed
// once per wave, one per lane, in fp64 (positions reach far past the 2^24 turns
// that fp32 resolves), and passed to the lanes through LDS.
#include "common.h"
#include "kernels.h"

namespace sas {

// 8 values from floats, rounded once
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* x) {
  if constexpr (sizeof(T) == 2) {
    *(uint4*)p = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                            pack_bf16x2(x[6], x[7]));
  } else {
    *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  }
}

// base^(-2 i / dh) of lane's pair i, and the axis whose position turns it
struct QkPair {
  double freq;  // turns per position
  int axis;
};
template <int DH>
__device__ __forceinline__ QkPair qk_pair(const QkArgs& P, int lane) {
  const int i = lane & (DH / 2 - 1);
  QkPair r;
  r.freq = exp2(-2.0 * (double)i / (double)DH * P.log2_base) * 0.15915494309189533577;  // / (2 pi)
  r.axis = P.axes == 1 || i < P.sec0 ? 0 : i < P.sec0 + P.sec1 ? 1 : 2;
  return r;
}
// cos and sin of the pair's angle: the fraction of a turn is taken in fp64, and what its
// rounding to fp32 leaves off (2^-26 of a turn, 10^-7 rad) turns the result by first order
__device__ __forceinline__ float2 qk_turn(const QkPair& pr, int pos) {
  const double a = (double)pos * pr.freq, t = a - rint(a);
  const float f = (float)t, rest = (float)(t - (double)f) * 6.28318530717958647693f;
  float s, c;
  sincospif(2.f * f, &s, &c);
  return make_float2(fmaf(-rest, s, c), fmaf(rest, c, s));
}

template <typename T>
__device__ __forceinline__ void load16(const T* p, int half, Vec8<T>& a, Vec8<T>& b) {
  a.load(p);
  b.load(p + half);
}

// sum over the DH / 16 lanes of a head
template <int DH>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int o = 1; o < DH / 16; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

constexpr int QK_PASSES = 4;  // head groups of a wave, all loaded before the first is used

// Unit: (row, QK_PASSES groups of heads); heads count q, then k, then v (cache).
template <typename T, int DH>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(QkArgs P, int parts, long long units) {
  constexpr int LPH = DH / 16, HPP = 64 / LPH;
  __shared__ __align__(16) float2 turn_s[4][DH / 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long unit = (long long)blockIdx.x * 4 + wave;
  if (unit >= units) return;
  const int row = (int)(unit / parts), part = (int)(unit % parts);
  const int c = lane % LPH, d0 = c * 8;
  const int heads = P.H + P.Hkv + (P.slot ? P.Hkv : 0);
  const int h0 = part * QK_PASSES * HPP + lane / LPH;
  Vec8<T> a[QK_PASSES], b[QK_PASSES];
#pragma unroll
  for (int u = 0; u < QK_PASSES; ++u) {
    const int h = min(h0 + u * HPP, heads - 1);
    const T* src = h < P.H             ? (const T*)P.q + row * P.qs + (long long)h * DH
                   : h < P.H + P.Hkv   ? (const T*)P.k + row * P.ks + (long long)(h - P.H) * DH
                                       : (const T*)P.v + row * P.vs + (long long)(h - P.H - P.Hkv) * DH;
    load16(src + d0, DH / 2, a[u], b[u]);
  }
  long long slot = -1;
  if (P.slot) {
    slot = P.slot[row];
    if (slot >= (long long)P.num_pages << P.ps_shift) slot = -1;
  }
  const QkPair pr = qk_pair<DH>(P, lane);
  const float2 t = qk_turn(pr, P.pos[(size_t)pr.axis * P.rows + row]);
  if (lane < DH / 2) turn_s[wave][lane] = t;
  wave_lds_fence();
  float cs[8], sn[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float2 x = turn_s[wave][d0 + e];
    cs[e] = x.x;
    sn[e] = x.y;
  }
  const size_t page = slot >= 0 ? (size_t)(slot >> P.ps_shift) : 0;
  const int at = slot >= 0 ? (int)(slot & ((1 << P.ps_shift) - 1)) : 0;
#pragma unroll
  for (int u = 0; u < QK_PASSES; ++u) {
    const int h = h0 + u * HPP;
    const bool isq = h < P.H, isk = !isq && h < P.H + P.Hkv, live = h < heads;
    const int hk = isk ? h - P.H : h - P.H - P.Hkv;
    float x[8], y[8];
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = a[u].get(e);
      y[e] = b[u].get(e);
      ss = fmaf(x[e], x[e], fmaf(y[e], y[e], ss));
    }
    const T* gain = (const T*)(isq ? P.gain_q : P.gain_k);
    ss = head_sum<DH>(ss);
    if (isq || isk) {
      if (gain) {
        Vec8<T> ga, gb;
        load16(gain + d0, DH / 2, ga, gb);
        const float r = rsqrtf(ss * (1.0f / DH) + P.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = x[e] * r * ga.get(e);
          y[e] = y[e] * r * gb.get(e);
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float n0 = x[e], n1 = y[e];
        x[e] = fmaf(n0, cs[e], -(n1 * sn[e]));
        y[e] = fmaf(n1, cs[e], n0 * sn[e]);
      }
    }
    if (!live) continue;
    if (isq || (isk && P.k_out)) {
      T* dst = isq ? (T*)P.q_out + ((size_t)row * P.H + h) * DH + d0 : (T*)P.k_out + ((size_t)row * P.Hkv + hk) * DH + d0;
      store8(dst, x);
      store8(dst + DH / 2, y);
    }
    if (!isq && slot >= 0) {
      T* dst = (T*)(isk ? P.k_pages : P.v_pages) + (((page * P.Hkv + hk) << P.ps_shift) + at) * DH + d0;
      store8(dst, x);
      store8(dst + DH / 2, y);
    }
  }
}

// Backward.  With dn the rotated-back gradient (the rotation's transpose) and
// r = rsqrt(mean x^2 + eps): dg += dn x r and dx = r (g dn - x r^2 mean(g dn x)).
// As many workgroups as stay resident walk the units (a row's group of heads) in
// runs of QK_RUN, so that a wave forms a row's angles once for several; it loads its
// next unit before it computes the current one.  Lanes keep the
// gains' gradients of their 16 dimensions in fp32 registers (a term for each of a lane's
// units: 43 at 16384 rows of 32/32 heads, where the result is 1.6e-7 off in norm) and
// leave one fp32 sum per workgroup, added in fp64 and a fixed order by qk_gain_sum_kernel.
// Measured at 16384 rows of 32/32 heads of 128 (bf16; 805 MB): 196 us with 1024
// workgroups of two units at a time and no loads ahead, 168 us with the 768 that are
// resident, 162 us with the next unit's loads ahead, 160 us (5.0 TB/s; a copy reaches
// 4.9) in runs of 2 (4: 167, one run a wave: 180).  Stores past the caches: 178 us, or
// 150 us if the forward before it, 5% slower, stores so too.
constexpr int QK_RUN = 2;
template <typename T>
struct QkBwdUnit {
  Vec8<T> a, b, da, db;  // x and its upstream gradient, both halves
  int row, h, pos;
};

template <typename T, int DH>
__global__ void __launch_bounds__(256) qk_norm_rope_bwd_kernel(QkArgs P, int parts, long long units) {
  constexpr int LPH = DH / 16, HPP = 64 / LPH;
  __shared__ __align__(16) float2 turn_s[4][DH / 2];
  __shared__ float gain_s[4][2][DH];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = lane % LPH, d0 = c * 8;
  const int heads = P.H + P.Hkv;
  const QkPair pr = qk_pair<DH>(P, lane);
  float dg[2][16];
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int e = 0; e < 16; ++e) dg[w][e] = 0.f;
  // (a unit past the end loads the last one again)
  auto load = [&](QkBwdUnit<T>& U, long long unit) {
    unit = min(unit, units - 1);
    U.row = (int)(unit / parts);
    U.h = (int)(unit % parts) * HPP + lane / LPH;
    const int h = min(U.h, heads - 1);
    const bool isq = h < P.H;
    const T* src = isq ? (const T*)P.q + U.row * P.qs + (long long)h * DH
                       : (const T*)P.k + U.row * P.ks + (long long)(h - P.H) * DH;
    const T* dsrc = isq ? (const T*)P.dq_out + ((size_t)U.row * P.H + h) * DH
                        : (const T*)P.dk_out + ((size_t)U.row * P.Hkv + (h - P.H)) * DH;
    U.pos = P.pos[(size_t)pr.axis * P.rows + U.row];
    load16(src + d0, DH / 2, U.a, U.b);
    load16(dsrc + d0, DH / 2, U.da, U.db);
  };
  const long long jump = ((long long)gridDim.x * 4 - 1) * QK_RUN;
  long long unit = ((long long)blockIdx.x * 4 + wave) * QK_RUN;
  QkBwdUnit<T> U, N;
  int turned = -1;  // the row whose angles LDS holds
  int left = QK_RUN;
  load(U, unit);
  while (unit < units) {
    unit += 1;
    if (--left == 0) {
      unit += jump;
      left = QK_RUN;
    }
    load(N, unit);
    if (U.row != turned) {
      const float2 t = qk_turn(pr, U.pos);
      wave_lds_fence();
      if (lane < DH / 2) turn_s[wave][lane] = t;
      wave_lds_fence();
      turned = U.row;
    }
    const bool isq = U.h < P.H, live = U.h < heads;
    float n0[8], n1[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 x = turn_s[wave][d0 + e];
      const float y0 = U.da.get(e), y1 = U.db.get(e);
      n0[e] = fmaf(y0, x.x, y1 * x.y);
      n1[e] = fmaf(y1, x.x, -(y0 * x.y));
    }
    const T* gain = (const T*)(isq ? P.gain_q : P.gain_k);
    Vec8<T> ga, gb;
    float ss = 0.f, sx = 0.f;
    if (gain) load16(gain + d0, DH / 2, ga, gb);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = U.a.get(e), y = U.b.get(e);
      ss = fmaf(x, x, fmaf(y, y, ss));
      if (gain) sx = fmaf(n0[e] * ga.get(e), x, fmaf(n1[e] * gb.get(e), y, sx));
    }
    ss = head_sum<DH>(ss);
    sx = head_sum<DH>(sx);
    if (gain) {
      const float r = rsqrtf(ss * (1.0f / DH) + P.eps);
      const float k = r * r * sx * (1.0f / DH);
      auto gains = [&](float* g) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          g[e] = fmaf(n0[e], U.a.get(e) * r, g[e]);
          g[8 + e] = fmaf(n1[e], U.b.get(e) * r, g[8 + e]);
        }
      };
      if (live) {
        if (isq) gains(dg[0]);
        else gains(dg[1]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = U.a.get(e), y = U.b.get(e);
        n0[e] = r * fmaf(n0[e], ga.get(e), -(x * k));
        n1[e] = r * fmaf(n1[e], gb.get(e), -(y * k));
      }
    }
    if (live) {
      T* dst = isq ? (T*)P.dq + ((size_t)U.row * P.H + U.h) * DH + d0
                   : (T*)P.dk + ((size_t)U.row * P.Hkv + (U.h - P.H)) * DH + d0;
      store8(dst, n0);
      store8(dst + DH / 2, n1);
    }
    U = N;
  }
  if (!P.part) return;
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float v = dg[w][e];
#pragma unroll
      for (int o = LPH; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
      if (lane < LPH) gain_s[wave][w][(e < 8 ? 0 : DH / 2) + d0 + (e & 7)] = v;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * DH; i += 256) {
    const float* g = &gain_s[0][0][0] + i;
    P.part[(size_t)blockIdx.x * 2 * DH + i] = (g[0] + g[2 * DH]) + (g[4 * DH] + g[6 * DH]);
  }
}

// dgain[w][d] = sum over the workgroups' sums, in fp64 and a fixed order: a
// workgroup takes 8 columns, a thread every 32nd row of one
__global__ void __launch_bounds__(256) qk_gain_sum_kernel(const float* part, int n, int dh, float* dq, float* dk) {
  __shared__ double s[32][8];
  const int col = blockIdx.x * 8 + (threadIdx.x & 7), j = threadIdx.x >> 3;
  double v = 0.0;
#pragma unroll 8
  for (int r = j; r < n; r += 32) v += (double)part[(size_t)r * 2 * dh + col];
  s[j][threadIdx.x & 7] = v;
  __syncthreads();
  if (threadIdx.x < 8) {
    for (int k = 1; k < 32; ++k) v += s[k][threadIdx.x];
    float* out = col < dh ? dq : dk;
    if (out) out[col < dh ? col : col - dh] = (float)v;
  }
}

// Summaries of the blocks that the chunk completes (mean of the block's keys as
// the pages hold them: fp64 sum in ascending order, rounded once; a position
// without a page adds zero), optionally projected.  A workgroup forms the prefix
// sum of the completed blocks over the sequences in LDS; a wave takes one (block,
// kv head) at a time, a lane dh / 64 dimensions.  Bound by waits: sums and table, a page,
// then the rows.  190 blocks of 4 kv heads of 128: 7.7 us; 64 rows together 7.4, 32 7.2
// (with more registers; blocks of 16 keys would load twice what they need).
template <typename T, int DH>
__global__ void __launch_bounds__(256) chunk_summary_kernel(BlockSumArgs P) {
  constexpr int NJ = DH / 64, STEP = 16;  // dimensions of a lane, rows loaded together (B >= 16)
  extern __shared__ __align__(16) unsigned char sum_lds[];
  int* const blk0 = (int*)sum_lds;  // [b] blocks completed before sequence i
  __shared__ int wsum[4];
  __shared__ float plain_s[4][DH];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (P.b + 255) / 256, i0 = min(tid * per, P.b), i1 = min(i0 + per, P.b);
  // blocks that sequence i completes, first block
  auto blocks = [&](int i, int& first) -> int {
    const int c = max(P.ctx_len[i], 0), e = max(P.kv_len[i], 0);
    first = c / P.B;
    return min(max(min(e / P.B, P.max_blocks) - first, 0), P.rows);
  };
  int n = 0, first;
  for (int i = i0; i < i1; ++i) n = min(n + blocks(i, first), P.rows);
  int x = n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x = min(x + y, P.rows);
  }
  if (lane == 63) wsum[wave] = x;
  __syncthreads();
  int at = __shfl_up(x, 1, 64), total = 0;
  if (lane == 0) at = 0;
  for (int w = 0; w < 4; ++w) {
    if (w < wave) at = min(at + wsum[w], P.rows);
    total = min(total + wsum[w], P.rows);
  }
  for (int i = i0; i < i1; ++i) {
    blk0[i] = at;
    at = min(at + blocks(i, first), P.rows);
  }
  __syncthreads();
  const long long items = (long long)total * P.Hkv;
  const int psm = (1 << P.ps_shift) - 1;
  for (long long it = (long long)blockIdx.x * 4 + wave; it < items; it += (long long)gridDim.x * 4) {
    const int g = (int)(it % P.Hkv), j = (int)(it / P.Hkv);
    int lo = 0, hi = P.b;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (blk0[mid] <= j) lo = mid;
      else hi = mid;
    }
    const int i = lo;
    (void)blocks(i, first);
    const int m = __builtin_amdgcn_readfirstlane(first + (j - blk0[i])), gs = __builtin_amdgcn_readfirstlane(g);
    double acc[NJ];
#pragma unroll
    for (int e = 0; e < NJ; ++e) acc[e] = 0.0;
    const int32_t* trow = P.table + (size_t)i * P.max_pages;
    for (int p0 = m * P.B; p0 < (m + 1) * P.B; p0 += 64) {
      // lane l holds the page of position p0 + l (-1: none, or past the block); the rows
      // are loaded STEP at a time, from clamped addresses
      const int pi = (p0 + lane) >> P.ps_shift;
      int page = trow[min(pi, P.max_pages - 1)];
      if (pi >= P.max_pages || page >= P.num_pages || p0 + lane >= (m + 1) * P.B) page = -1;
      for (int q0 = 0; q0 < 64 && p0 + q0 < (m + 1) * P.B; q0 += STEP) {
        struct Row {
          T v[NJ];
        } row[STEP];
        bool ok[STEP];
#pragma unroll
        for (int u = 0; u < STEP; ++u) {
          const int pg = __builtin_amdgcn_readlane(page, q0 + u);
          ok[u] = pg >= 0;
          const T* at = (const T*)P.k_pages + ((((size_t)max(pg, 0) * P.Hkv + gs) << P.ps_shift) + ((p0 + q0 + u) & psm)) * DH;
          row[u] = *(const Row*)(at + lane * NJ);
        }
#pragma unroll
        for (int u = 0; u < STEP; ++u)
#pragma unroll
          for (int e = 0; e < NJ; ++e) acc[e] += ok[u] ? (double)Act<T>::to_f32(row[u].v[e]) : 0.0;
      }
    }
    T r[NJ];
#pragma unroll
    for (int e = 0; e < NJ; ++e) r[e] = Act<T>::from_f64(acc[e] / (double)P.B);
    T* dst = (T*)P.k_summary + (((size_t)i * P.Hkv + g) * P.max_blocks + m) * DH;
    if (!P.w_gk) {
#pragma unroll
      for (int e = 0; e < NJ; ++e) dst[lane * NJ + e] = r[e];
      continue;
    }
    wave_lds_fence();
#pragma unroll
    for (int e = 0; e < NJ; ++e) plain_s[wave][lane * NJ + e] = Act<T>::to_f32(r[e]);
    wave_lds_fence();
#pragma unroll
    for (int e = 0; e < NJ; ++e) {
      const T* w = (const T*)P.w_gk + ((size_t)g * DH + lane * NJ + e) * DH;
      double s = 0.0;
      for (int d = 0; d < DH; ++d) s = fma((double)Act<T>::to_f32(w[d]), (double)plain_s[wave][d], s);
      dst[lane * NJ + e] = Act<T>::from_f64(s);
    }
  }
}

hipError_t launch_qk_norm_rope(int dtype, const QkArgs& a, hipStream_t s) {
  const int hpp = 1024 / a.dh, heads = a.H + a.Hkv * (a.slot ? 2 : 1);
  const int parts = cdiv(heads, hpp * QK_PASSES);
  const long long units = (long long)a.rows * parts;
  const unsigned grid = (unsigned)((units + 3) / 4);
  if (dtype == SAS_BF16) {
    if (a.dh == 128) qk_norm_rope_kernel<bf16_t, 128><<<grid, 256, 0, s>>>(a, parts, units);
    else qk_norm_rope_kernel<bf16_t, 64><<<grid, 256, 0, s>>>(a, parts, units);
  } else {
    if (a.dh == 128) qk_norm_rope_kernel<float, 128><<<grid, 256, 0, s>>>(a, parts, units);
    else qk_norm_rope_kernel<float, 64><<<grid, 256, 0, s>>>(a, parts, units);
  }
  return hipGetLastError();
}

hipError_t launch_qk_norm_rope_backward(int dtype, const QkArgs& a, hipStream_t s) {
  const int hpp = 1024 / a.dh, parts = cdiv(a.H + a.Hkv, hpp);
  const long long units = (long long)a.rows * parts;
  const int grid = (int)std::min<long long>(QK_BWD_GROUPS, (units + 3) / 4);
  if (dtype == SAS_BF16) {
    if (a.dh == 128) qk_norm_rope_bwd_kernel<bf16_t, 128><<<grid, 256, 0, s>>>(a, parts, units);
    else qk_norm_rope_bwd_kernel<bf16_t, 64><<<grid, 256, 0, s>>>(a, parts, units);
  } else {
    if (a.dh == 128) qk_norm_rope_bwd_kernel<float, 128><<<grid, 256, 0, s>>>(a, parts, units);
    else qk_norm_rope_bwd_kernel<float, 64><<<grid, 256, 0, s>>>(a, parts, units);
  }
  if (a.part) qk_gain_sum_kernel<<<2 * a.dh / 8, 256, 0, s>>>(a.part, grid, a.dh, a.dgain_q, a.dgain_k);
  return hipGetLastError();
}

hipError_t launch_chunk_summaries(int dtype, const BlockSumArgs& a, hipStream_t s) {
  // every sequence completes at most one block more than its rows hold
  const long long most = ((long long)a.rows / a.B + std::min(a.b, a.rows)) * a.Hkv;
  const unsigned grid = (unsigned)std::max<long long>(1, std::min<long long>(2048, (most + 3) / 4));
  const size_t lds = (size_t)a.b * 4;
  if (dtype == SAS_BF16) {
    if (a.dh == 128) chunk_summary_kernel<bf16_t, 128><<<grid, 256, lds, s>>>(a);
    else chunk_summary_kernel<bf16_t, 64><<<grid, 256, lds, s>>>(a);
  } else {
    if (a.dh == 128) chunk_summary_kernel<float, 128><<<grid, 256, lds, s>>>(a);
    else chunk_summary_kernel<float, 64><<<grid, 256, lds, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace sas
