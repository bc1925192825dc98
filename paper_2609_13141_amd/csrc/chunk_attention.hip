// Causal attention of a chunk of new tokens over the paged cache.
//
// Row j of sequence i's chunk (m rows, kv_len keys cached, the chunk's own
// among them) stands at position t = kv_len - m + j and attends the mapped
// positions up to t: o = sum_p softmax(sm q.k_p) v_p in one pass over the keys
// with a running maximum and sum.
//
// The lengths are device memory, so the work is divided on the device: a tile
// is 128 rows (128 / G consecutive tokens x the G heads of a kv head, which
// read the same keys), and chunk_plan_kernel cuts the tiles' key ranges into
// parts of at most C key tiles, C the average work of a resident workgroup;
// parts are merged by chunk_combine_kernel.  Workgroups take the jobs from
// eight queues, one per XCD, each a contiguous share, so that the tiles of one
// (sequence, kv head) read its keys from one L2.
//
// The tile loop is that of the prefill kernel (S^T = K Q^T, P^T fed back from
// registers as the B operand of O^T = V^T P^T) with rows found through the
// block table: a wave holds the page of key l of the next tile in lane l, one
// load per tile, and gives it to the copying lanes with a permute.
#include <float.h>
#include <stdint.h>

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace sas {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

typedef __attribute__((address_space(3))) void chunk_lds_t;

// Keys of a tile: 64 in bf16, 32 in fp32 (the same bytes).
template <typename T> struct ChunkTile;
template <> struct ChunkTile<bf16_t> { static constexpr int KEYS = 64; };
template <> struct ChunkTile<float> { static constexpr int KEYS = 32; };

// position of 16-byte chunk c of tile row r (bank-conflict-free for the reads below)
template <typename T, int DH>
__device__ __forceinline__ int chunk_swz(int r) {
  if constexpr (sizeof(T) == 2) return lds_swz<DH>(r);
  else return r & 15;
}

// Sequence i's rows and keys, clamped so that no array contents can lead out of range.
struct ChunkSeq {
  int r0, m;    // first row, rows
  int base;     // position of the first row (may be negative: such rows attend nothing)
  int keys;     // cached positions that the block table covers
};
__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkArgs& P, int i) {
  ChunkSeq s;
  s.r0 = min(max(P.row_start[i], 0), P.rows);
  s.m = min(max(P.row_start[i + 1], s.r0), P.rows) - s.r0;
  const int kv = max(P.kv_len[i], 0);
  s.base = kv - s.m;
  s.keys = (int)min((long long)kv, (long long)P.max_pages << P.ps_shift);
  return s;
}

// largest i in [0, n) with base[i] <= x, by the 64 lanes of a wave (base[0] <= x, n <= 4096)
__device__ __forceinline__ int wave_find(const int* base, int n, int x, int lane) {
  const int step = (n + 63) / 64;
  const int k = lane * step;
  const unsigned long long a = __builtin_amdgcn_ballot_w64(k < n && base[min(k, n - 1)] <= x);
  const int lo = (63 - __builtin_clzll(a)) * step;
  if (step == 1) return lo;
  const unsigned long long c = __builtin_amdgcn_ballot_w64(lane < step && lo + lane < n && base[min(lo + lane, n - 1)] <= x);
  return lo + 63 - __builtin_clzll(c);
}

// sum over the workgroup's 1024 threads of v, and the sum before this thread (s: 17 values of LDS)
__device__ __forceinline__ long long scan1024(long long v, long long* s, long long& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) s[wave] = x;
  __syncthreads();
  long long before = 0, tot = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    if (w < wave) before += s[w];
    tot += s[w];
  }
  total = tot;
  return before + x - v;
}

// One workgroup: divides the work (see above) and clears the job queues.
// head[0] = jobs, head[1] = C, head[8 + x] = the next job of XCD x's share.
__global__ void __launch_bounds__(1024) chunk_plan_kernel(ChunkArgs P, int keys_per_tile, int want_parts) {
  __shared__ long long s[17];
  const int tid = threadIdx.x, per = (P.b + 1023) / 1024;
  const int qpt = 128 / (P.H / P.Hkv);
  long long W = 0, total;
  for (int u = 0; u < per; ++u) {
    const int i = tid * per + u;
    if (i >= P.b) break;
    const ChunkSeq q = chunk_seq(P, i);
    W += (long long)P.Hkv * ((q.m + qpt - 1) / qpt) * ((q.keys + keys_per_tile - 1) / keys_per_tile);
  }
  (void)scan1024(W, s, total);
  // at most 2 W / C parts in all of the divided tiles: they fit the scratch
  long long C = max((long long)CHUNK_MIN_TILES, (total + want_parts - 1) / want_parts);
  C = P.part_slots > 0 ? max(C, (2 * total + P.part_slots - 1) / P.part_slots) : 0x7fffffffll;
  long long jobs = 0, slots = 0;
  for (int u = 0; u < per; ++u) {
    const int i = tid * per + u;
    if (i >= P.b) break;
    const ChunkSeq q = chunk_seq(P, i);
    const long long nk = (q.keys + keys_per_tile - 1) / keys_per_tile;
    const long long parts = max(1ll, (nk + C - 1) / C);
    const long long j = (long long)P.Hkv * ((q.m + qpt - 1) / qpt) * parts;
    jobs += j;
    if (parts > 1) slots += j;
  }
  long long njobs, nslots;
  long long j0 = scan1024(jobs, s, njobs), s0 = scan1024(slots, s, nslots);
  for (int u = 0; u < per; ++u) {
    const int i = tid * per + u;
    if (i >= P.b) break;
    const ChunkSeq q = chunk_seq(P, i);
    const long long nk = (q.keys + keys_per_tile - 1) / keys_per_tile;
    const long long parts = max(1ll, (nk + C - 1) / C);
    const long long j = (long long)P.Hkv * ((q.m + qpt - 1) / qpt) * parts;
    P.job_base[i] = (int)j0;
    P.seq_parts[i] = make_int2((int)parts, (int)s0);
    j0 += j;
    if (parts > 1) s0 += j;
  }
  if (tid == 0) {
    P.head[0] = (int)njobs;
    P.head[1] = nslots > 0;
  }
  if (tid < ATTN_XCDS) P.head[8 + tid] = (int)(njobs * tid / ATTN_XCDS);
}

template <typename T, int DH>
__device__ __forceinline__ void chunk_job(const ChunkArgs& P, const int seq, const int rel) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int KEYS = ChunkTile<T>::KEYS, NST = KEYS / 32;
  constexpr int CH = DH * (int)sizeof(T) / 16;  // 16-byte pieces of a row
  constexpr int RB = DH * (int)sizeof(T);       // bytes of a row
  constexpr int TB = KEYS * RB;                 // bytes of a tile
  constexpr int NL = KEYS * CH / 256;           // pieces of K (and of V) per thread and tile
  // two buffers of K and V (4 TB bytes; dynamic, because the compiler makes every read
  // of a static array wait for the direct-to-LDS loads in flight)
  extern __shared__ __align__(16) unsigned char tiles[];
  __shared__ unsigned long long bad_s;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lk = lane >> 5;
  const int G = P.H / P.Hkv, QPT = 128 / G;
  const ChunkSeq S = chunk_seq(P, seq);
  const int2 sp = P.seq_parts[seq];
  const int ntile = (S.m + QPT - 1) / QPT;
  const int part = rel % sp.x, tile = ntile - 1 - (rel / sp.x) % ntile, g = rel / sp.x / ntile;
  const int slot = sp.x > 1 ? sp.y + rel : -1;

  const int qrow = wave * 32 + lr;
  const int pl = qrow / G, h = g * G + (qrow - pl * G);
  const bool qvalid = pl < QPT && tile * QPT + pl < S.m;
  const int t0 = S.base + tile * QPT;                            // position of the tile's first row
  const int t_hi = S.base + min(tile * QPT + QPT, S.m) - 1;      // and of its last
  const int t = qvalid ? t0 + pl : -1;
  const size_t row = (size_t)S.r0 + tile * QPT + pl;
  const bool wave_live = __builtin_amdgcn_ballot_w64(qvalid) != 0;
  // this part's key tiles
  const int nkt = (min(max(t_hi + 1, 0), S.keys) + KEYS - 1) / KEYS;
  const int per = (nkt + sp.x - 1) / sp.x;
  const int tlo = part * per, tend = min(tlo + per, nkt);

  // Q^T as the B operand of S^T = K Q^T.  bf16: lane supplies dimensions
  // 16 ks + 8 lk + 0..7; fp32: 8 ks + 4 lk + e for step (ks, e)
  constexpr int NQ = BF ? DH / 16 : DH / 8;
  uint4 qb[NQ];
  {
    const T* qp = (const T*)P.Q + (row * P.H + h) * DH;
#pragma unroll
    for (int ks = 0; ks < NQ; ++ks)
      qb[ks] = qvalid ? *(const uint4*)(qp + (BF ? ks * 16 + lk * 8 : ks * 8 + lk * 4)) : make_uint4(0, 0, 0, 0);
  }

  floatx16_t o[DH / 32];
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[dt][v] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const float qk_scale = P.sm_scale * LOG2E;

  const int32_t* trow = P.table + (size_t)seq * P.max_pages;
  const int psm = (1 << P.ps_shift) - 1;
  // the page of key `lane` of tile kt (-1: no such key, or unmapped)
  auto load_pages = [&](int kt) -> int {
    const int p = kt * KEYS + (lane & (KEYS - 1));
    const int page = trow[min(p >> P.ps_shift, P.max_pages - 1)];
    return p < S.keys && page >= 0 && page < P.num_pages ? page : -1;
  };
  // K and V rows of tile kt into buffer buf; keys without a page read page 0
  auto load_tile = [&](int kt, int pg, int buf) {
    unsigned char* tb = tiles + buf * 2 * TB;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int p = (wave * NL + i) * 64 + lane, r = p / CH, c = (p % CH) ^ chunk_swz<T, DH>(r);
      const int page = max(__shfl(pg, r, 64), 0);
      const size_t off = ((((size_t)page * P.Hkv + g) << P.ps_shift) + ((kt * KEYS + r) & psm)) * DH + c * (16 / sizeof(T));
      unsigned char* d = tb + (wave * NL + i) * 1024;
      __builtin_amdgcn_global_load_lds((const void*)((const T*)P.k_pages + off), (chunk_lds_t*)d, 16, 0, 0);
      __builtin_amdgcn_global_load_lds((const void*)((const T*)P.v_pages + off), (chunk_lds_t*)(d + TB), 16, 0, 0);
    }
  };
  constexpr unsigned long long ALL = KEYS == 64 ? ~0ull : 0xffffffffull;
  auto valid_mask = [&](int pg) { return __builtin_amdgcn_ballot_w64(pg >= 0) & ALL; };

  // byte offsets of this lane's operands in a tile: K row lr (+ 32 st), chunk 2 ks + lk;
  // bf16 V columns by transposing reads (rows 4 lk + 8 half + (lane % 16) / 4)
  uint32_t o_row = lr * RB + ((lk ^ chunk_swz<T, DH>(lr)) << 4);
  uint32_t o_tr[2] = {0, 0};
  if constexpr (BF) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int r = 4 * lk + 8 * hf + ((lane & 15) >> 2);
      o_tr[hf] = r * RB + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ chunk_swz<T, DH>(r)) << 4) + (lane & 1) * 8;
    }
  }

  int kt = tlo, buf = 0;
  int pg = -1;
  unsigned long long vcur = 0;
  if (kt < tend) {
    pg = load_pages(kt);
    load_tile(kt, pg, 0);
    vcur = valid_mask(pg);
    pg = load_pages(kt + 1);
  }
  for (; kt < tend; ++kt, buf ^= 1) {
    // this wave's loads of the tile are done; after the barrier everyone's are,
    // and every wave is done with the other buffer
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const int k0 = kt * KEYS;
    unsigned char* const tb = tiles + buf * 2 * TB;
    asm volatile("" : "+v"(o_row), "+v"(o_tr[0]), "+v"(o_tr[1]));  // (formed anew per tile: kept, they would spill)
    const unsigned long long vnext = valid_mask(pg);
    if (kt + 1 < tend) {
      load_tile(kt + 1, pg, buf ^ 1);
      pg = load_pages(kt + 2);
    }
    const bool diag = k0 + KEYS - 1 > t0, gaps = vcur != ALL;
    if (diag || gaps) {
      // A product with P = 0 would turn an infinite or NaN value of a key that a row
      // does not attend into NaN.  Values of keys without a page are zeroed; infinite
      // and NaN elements of the others are added to the rows that do attend them (the
      // sum is not finite whatever their weight) and then zeroed too.
      if (tid == 0) bad_s = 0;
      lds_barrier();
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int r = ((wave * NL + i) * 64 + lane) / CH;
        uint4* pv = (uint4*)(tb + TB + (wave * NL + i) * 1024 + lane * 16);
        if (!((vcur >> r) & 1)) {
          *pv = make_uint4(0, 0, 0, 0);
        } else {
          const uint4 u = *pv;
          const uint32_t w[4] = {u.x, u.y, u.z, u.w};
          bool bad = false;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            bad = bad || (w[e] & 0x7f800000u) == 0x7f800000u;
            if constexpr (BF) bad = bad || (w[e] & 0x7f80u) == 0x7f80u;
          }
          if (bad) atomicOr(&bad_s, 1ull << r);
        }
      }
      lds_barrier();
      unsigned long long bm = bad_s;
      if (bm) {
        for (; bm; bm &= bm - 1) {
          const int r = __builtin_ctzll(bm);
          if (k0 + r > t) continue;
#pragma unroll
          for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const int d = dt * 32 + 8 * (v >> 2) + 4 * lk + (v & 3);
              const int c = d * (int)sizeof(T) / 16;
              const T x = *(const T*)(tb + TB + r * RB + ((c ^ chunk_swz<T, DH>(r)) << 4) + d * sizeof(T) % 16);
              const float f = Act<T>::to_f32(x);
              if (!(fabsf(f) < INFINITY)) o[dt][v] += f;
            }
        }
        lds_barrier();
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          T* pv = (T*)(tb + TB + (wave * NL + i) * 1024 + lane * 16);
#pragma unroll
          for (int e = 0; e < 16 / (int)sizeof(T); ++e)
            if (!(fabsf(Act<T>::to_f32(pv[e])) < INFINITY)) pv[e] = 0;
        }
        lds_barrier();
      }
    }
    if (wave_live) {
      __builtin_amdgcn_s_setprio(2);
      floatx16_t s[NST];
#pragma unroll
      for (int st = 0; st < NST; ++st)
#pragma unroll
        for (int v = 0; v < 16; ++v) s[st][v] = 0.f;
      if constexpr (BF) {
        bf16x8_t ka0 = *(const bf16x8_t*)(tb + o_row), ka1 = *(const bf16x8_t*)(tb + o_row + 32 * RB);
#pragma unroll
        for (int ks = 0; ks < DH / 16; ++ks) {
          bf16x8_t kn0 = ka0, kn1 = ka1;
          if (ks + 1 < DH / 16) {
            const unsigned char* kf = tb + (o_row ^ ((ks + 1) << 5));
            kn0 = *(const bf16x8_t*)kf;
            kn1 = *(const bf16x8_t*)(kf + 32 * RB);
          }
          s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka0, *(const bf16x8_t*)&qb[ks], s[0], 0, 0, 0);
          s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka1, *(const bf16x8_t*)&qb[ks], s[1], 0, 0, 0);
          ka0 = kn0;
          ka1 = kn1;
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
        for (int ks = 0; ks < DH / 16; ++ks) {
          if (ks + 1 < DH / 16) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < DH / 8; ++ks) {
          const floatx4_t ka = *(const floatx4_t*)(tb + (o_row ^ (ks << 5)));
          const floatx4_t qv = *(const floatx4_t*)&qb[ks];
#pragma unroll
          for (int e = 0; e < 4; ++e) s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(ka[e], qv[e], s[0], 0, 0, 0);
        }
      }
      __builtin_amdgcn_s_setprio(0);
      if (diag) {
#pragma unroll
        for (int st = 0; st < NST; ++st)
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (k0 + st * 32 + 8 * (v >> 2) + 4 * lk + (v & 3) > t) s[st][v] = -INFINITY;
      }
      if (gaps) {
        const unsigned long long vm = vcur >> (4 * lk);
#pragma unroll
        for (int st = 0; st < NST; ++st)
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (!((vm >> (st * 32 + 8 * (v >> 2) + (v & 3))) & 1)) s[st][v] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int st = 0; st < NST; ++st)
#pragma unroll
        for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[st][v]);
      mx *= qk_scale;  // the scale is positive
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      // The reference m_run moves only when a logit exceeds it by more than 8 (log2
      // units): any reference gives the same sums, and the accumulators are rescaled
      // on few tiles.
      const bool upd = mx > m_run + 8.f;
      float alpha = 1.f;
      if (upd) {
        // (nothing is summed yet where m_run is -inf)
        alpha = m_run == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - mx);
        m_run = mx;
      }
      const float bias = m_run == -INFINITY ? 0.f : -m_run;
      float rs4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NST; ++st)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[st][v], qk_scale, bias));
          rs4[v & 3] += p;
          s[st][v] = p;
        }
      float rs = (rs4[0] + rs4[1]) + (rs4[2] + rs4[3]);
      rs += __shfl_xor(rs, 32, 64);
      l_run = l_run * alpha + rs;
      if (__builtin_amdgcn_ballot_w64(upd) != 0) {
#pragma unroll
        for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[dt][v] *= alpha;
      }
      __builtin_amdgcn_s_setprio(2);
      if constexpr (BF) {
        // P is rounded to bf16 for the matrix instruction (relative error 2^-9 a
        // weight, averaged over the keys; the sum l keeps the fp32 weights)
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          const int st = ks >> 1, v0 = 8 * (ks & 1);
          uint4 pu;
          pu.x = pack_bf16x2(s[st][v0 + 0], s[st][v0 + 1]);
          pu.y = pack_bf16x2(s[st][v0 + 2], s[st][v0 + 3]);
          pu.z = pack_bf16x2(s[st][v0 + 4], s[st][v0 + 5]);
          pu.w = pack_bf16x2(s[st][v0 + 6], s[st][v0 + 7]);
          const bf16x8_t pb = *(const bf16x8_t*)&pu;
#pragma unroll
          for (int dt = 0; dt < DH / 32; ++dt) {
            const uint2 lo = lds_read_tr(tb + TB + (o_tr[0] ^ (dt << 6)) + ks * 16 * RB);
            const uint2 hi = lds_read_tr(tb + TB + (o_tr[1] ^ (dt << 6)) + ks * 16 * RB);
            const uint4 vu = make_uint4(lo.x, lo.y, hi.x, hi.y);
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8_t*)&vu, pb, o[dt], 0, 0, 0);
          }
        }
      } else {
        // element v of P^T holds keys 8 (v / 4) + 4 lk + v % 4: step v multiplies those two keys
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = 8 * (v >> 2) + 4 * lk + (v & 3);
#pragma unroll
          for (int dt = 0; dt < DH / 32; ++dt) {
            const int c = dt * 8 + (lr >> 2);
            const float x = *(const float*)(tb + TB + r * RB + ((c ^ chunk_swz<T, DH>(r)) << 4) + (lr & 3) * 4);
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, s[0][v], o[dt], 0, 0, 0);
          }
        }
      }
      __builtin_amdgcn_s_setprio(0);
    }
    vcur = vnext;
  }

  if (slot >= 0) {  // a part: unnormalized sums and (max, sum) per row
    if (!qvalid) return;
    float* po = P.part_o + ((size_t)slot * 128 + qrow) * DH;
#pragma unroll
    for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4)
        *(float4*)(po + dt * 32 + 8 * v4 + 4 * lk) =
            make_float4(o[dt][4 * v4 + 0], o[dt][4 * v4 + 1], o[dt][4 * v4 + 2], o[dt][4 * v4 + 3]);
    if (lk == 0) *(float2*)(P.part_ml + ((size_t)slot * 128 + qrow) * 2) = make_float2(m_run, l_run);
    return;
  }
  if (!qvalid) return;
  const float inv_l = l_run == 0.f ? 0.f : 1.0f / l_run;
  T* op = (T*)P.O + (row * P.H + h) * DH;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int v4 = 0; v4 < 4; ++v4) {
      const int d0 = dt * 32 + 8 * v4 + 4 * lk;
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = l_run == 0.f ? 0.f : o[dt][4 * v4 + e] * inv_l;
      if constexpr (BF) *(uint2*)(op + d0) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
      else *(float4*)(op + d0) = make_float4(x[0], x[1], x[2], x[3]);
    }
  if (P.lse && lk == 0) P.lse[row * P.H + h] = l_run == 0.f ? -INFINITY : (m_run + log2f(l_run)) * LN2;
}

// Jobs from the XCD's queue, then from the next XCDs': a share is a contiguous
// range of jobs, and every workgroup leaves once all eight are drained.
template <typename T, int DH>
__global__ void __launch_bounds__(256, 2) chunk_attn_kernel(ChunkArgs P) {
  __shared__ int2 job_s;
  const int lane = threadIdx.x & 63;
  const int njobs = P.head[0];
  int drained = 0;
  for (;;) {
    __syncthreads();  // every thread has finished the previous job and read job_s
    if (threadIdx.x < 64) {
      int job = -1;
      while (drained < ATTN_XCDS) {
        const int x = (blockIdx.x + drained) % ATTN_XCDS;
        const int end = (int)((long long)njobs * (x + 1) / ATTN_XCDS);
        int j = 0;
        if (lane == 0) j = atomicAdd(&P.head[8 + x], 1);
        j = __builtin_amdgcn_readfirstlane(j);
        if (j < end) {
          job = j;
          break;
        }
        ++drained;
      }
      int2 r = make_int2(-1, 0);
      if (job >= 0) {
        r.x = wave_find(P.job_base, P.b, job, lane);
        r.y = job - P.job_base[r.x];
      }
      if (lane == 0) job_s = r;
    }
    __syncthreads();
    const int2 r = job_s;
    if (r.x < 0) break;
    chunk_job<T, DH>(P, __builtin_amdgcn_readfirstlane(r.x), __builtin_amdgcn_readfirstlane(r.y));
  }
}

// Merge of divided tiles: a workgroup takes rows in turn, a thread 8 dimensions of a head.
template <typename T, int DH>
__global__ void __launch_bounds__(256) chunk_combine_kernel(ChunkArgs P) {
  if (P.head[1] == 0) return;
  constexpr int C8 = DH / 8;
  const int lane = threadIdx.x & 63;
  const int G = P.H / P.Hkv, QPT = 128 / G;
  for (int r = blockIdx.x; r < P.rows; r += gridDim.x) {
    if (r < P.row_start[0] || r >= P.row_start[P.b]) continue;
    const int i = __builtin_amdgcn_readfirstlane(wave_find(P.row_start, P.b, r, lane));
    const int2 sp = P.seq_parts[i];
    if (sp.x <= 1) continue;
    const ChunkSeq S = chunk_seq(P, i);
    const int j = r - S.r0;
    if (j >= S.m) continue;
    const int ntile = (S.m + QPT - 1) / QPT, tile = j / QPT, pl = j - tile * QPT;
    for (int idx = threadIdx.x; idx < P.H * C8; idx += 256) {
      const int h = idx / C8, c8 = idx % C8, g = h / G;
      const size_t s0 = (size_t)sp.y + (size_t)(g * ntile + (ntile - 1 - tile)) * sp.x;
      const int qrow = pl * G + (h - g * G);
      float mx = -INFINITY;
      for (int p = 0; p < sp.x; ++p) mx = fmaxf(mx, P.part_ml[((s0 + p) * 128 + qrow) * 2]);
      const float mu = mx == -INFINITY ? 0.f : mx;
      float l = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      for (int p = 0; p < sp.x; ++p) {
        const size_t sr = (s0 + p) * 128 + qrow;
        const float2 ml = *(const float2*)(P.part_ml + sr * 2);
        const float w = __builtin_amdgcn_exp2f(ml.x - mu);
        const float4 a = *(const float4*)(P.part_o + sr * DH + c8 * 8);
        const float4 b = *(const float4*)(P.part_o + sr * DH + c8 * 8 + 4);
        if (ml.y == 0.f) continue;  // nothing attended in this part
        l += ml.y * w;
        acc[0] += a.x * w;
        acc[1] += a.y * w;
        acc[2] += a.z * w;
        acc[3] += a.w * w;
        acc[4] += b.x * w;
        acc[5] += b.y * w;
        acc[6] += b.z * w;
        acc[7] += b.w * w;
      }
      const float inv_l = l == 0.f ? 0.f : 1.0f / l;
      T* op = (T*)P.O + ((size_t)r * P.H + h) * DH + c8 * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) op[e] = Act<T>::from_f32(acc[e] * inv_l);
      if (P.lse && c8 == 0) P.lse[(size_t)r * P.H + h] = l == 0.f ? -INFINITY : (mu + log2f(l)) * LN2;
    }
  }
}

hipError_t launch_chunk_attention(int dtype, const ChunkArgs& a, hipStream_t s) {
  const int G = a.H / a.Hkv, qpt = 128 / G;
  const int keys = dtype == SAS_BF16 ? 64 : 32;
  const size_t lds = (size_t)512 * a.dh;  // two buffers of K and V tiles
  void (*kern)(ChunkArgs);
  void (*comb)(ChunkArgs);
  if (dtype == SAS_BF16) {
    kern = a.dh == 128 ? chunk_attn_kernel<bf16_t, 128> : chunk_attn_kernel<bf16_t, 64>;
    comb = a.dh == 128 ? chunk_combine_kernel<bf16_t, 128> : chunk_combine_kernel<bf16_t, 64>;
  } else {
    kern = a.dh == 128 ? chunk_attn_kernel<float, 128> : chunk_attn_kernel<float, 64>;
    comb = a.dh == 128 ? chunk_combine_kernel<float, 128> : chunk_combine_kernel<float, 64>;
  }
  const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  const int res = resident_workgroups(kern, 256, lds);
  if (res <= 0) return hipErrorInvalidValue;
  // the most jobs that there can be: tiles of every sequence, in parts of the least length
  const long long tiles = ((long long)a.rows / qpt + std::min(a.b, a.rows)) * a.Hkv;
  const long long max_keys = std::min((long long)a.max_pages << a.ps_shift, 0x7fffffffll);
  const long long parts = a.part_slots > 0 ? (max_keys + (long long)keys * CHUNK_MIN_TILES - 1) / ((long long)keys * CHUNK_MIN_TILES) : 1;
  const long long most = parts < res ? tiles * parts : res;
  chunk_plan_kernel<<<1, 1024, 0, s>>>(a, keys, res);
  kern<<<(unsigned)std::min<long long>(res, most), 256, lds, s>>>(a);
  if (a.part_slots > 0) comb<<<(unsigned)std::min(a.rows, 2048), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace sas
