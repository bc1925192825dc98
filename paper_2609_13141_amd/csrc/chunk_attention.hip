// Causal attention of a chunk of new tokens over the paged cache.
//
// Row j of sequence i's chunk (m rows, kv_len keys cached, the chunk's own
// among them) stands at position t = kv_len - m + j and attends the mapped
// positions up to t: o = sum_p softmax(sm q.k_p) v_p in one pass over the keys
// with a running maximum and sum.
//
// The lengths are device memory, so the work is divided on the device: a tile
// is 128 rows (128 / G consecutive tokens x the G heads of a kv head, which
// read the same keys), and the tiles' key ranges are cut into parts of at most C
// key tiles (chunk_part_length), merged by chunk_combine_kernel.  Jobs are
// numbered so that those that read the same keys follow each other, and each XCD
// takes a contiguous share, one job a workgroup where they all fit the chip at
// once, through a queue per XCD otherwise.  Up to 64 sequences every workgroup
// forms the division itself, a lane a sequence; more take a kernel of their own.
//
// The tile loop is that of the prefill kernel (S^T = K Q^T, P^T fed back from
// registers as the B operand of O^T = V^T P^T) with rows found through the
// block table: a wave loads the entries of a tile's keys once, a tile ahead, and
// copies the rows of a page from one scalar address.
#include <float.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace sas {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

typedef __attribute__((address_space(3))) void chunk_lds_t;

// Keys of a tile: 64 in bf16, 32 in fp32 (the same bytes).  LEAST: tiles of the shortest
// part.  An fp32 tile takes 2.9 us, more than another part's merge: 3 sequences of up to 50
// new tokens over up to 200 keys take 14.8 us with parts of one tile and 16.3 with two.  A
// bf16 tile takes less, and parts of one tile gained nothing.
template <typename T> struct ChunkTile;
template <> struct ChunkTile<bf16_t> { static constexpr int KEYS = 64, LEAST = 2; };
template <> struct ChunkTile<float> { static constexpr int KEYS = 32, LEAST = 1; };

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

__device__ __forceinline__ unsigned long long uniform64(unsigned long long x) {
  return (unsigned long long)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x) |
         (unsigned long long)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(x >> 32)) << 32;
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

// The work of one sequence: (tile, kv head) pairs, key tiles of each (the last
// tile's count: earlier ones have up to 128 / KEYS fewer), rows of a tile's part.
struct ChunkWork {
  int units, nk, prow;
};
__device__ __forceinline__ ChunkWork chunk_work(const ChunkArgs& P, const ChunkSeq& q, int keys_per_tile) {
  const int G = P.H / P.Hkv, qpt = CHUNK_ROWS / G;
  ChunkWork w;
  w.units = P.Hkv * ((q.m + qpt - 1) / qpt);
  w.nk = (q.keys + keys_per_tile - 1) / keys_per_tile;
  w.prow = min(q.m, qpt) * G;
  return w;
}
__device__ __forceinline__ int chunk_parts(int nk, int C) { return max(1, (int)(((uint32_t)nk + (uint32_t)C - 1) / (uint32_t)C)); }

// The length C of a part, in key tiles.  With fewer (tile, head) pairs than resident
// workgroups, the least C whose parts still fit them: one round of jobs, none longer
// than it has to be.  With more, a part is the average work of a workgroup, which
// only cuts tiles far longer than the others.  A divided tile has at most 2 nk / C
// parts, so that C >= 2 sum(units nk prow) / part_rows keeps them inside the scratch.
// sum(f): the sum over all sequences of f of their work, the same in every thread (in
// fp64, exact up to 2^53; a sequence counts for at most 2^20 parts).
template <typename Sum>
__device__ __forceinline__ int chunk_part_length(const ChunkArgs& P, int least_tiles, int res, Sum sum) {
  if (P.part_rows <= 0) return 0x7fffffff;
  const double U = sum([](const ChunkWork& w) { return (double)w.units; });
  const double W = sum([](const ChunkWork& w) { return (double)w.units * w.nk; });
  const double R = sum([](const ChunkWork& w) { return (double)w.units * w.nk * w.prow; });
  const double least = fmax((double)least_tiles, ceil(2.0 * R / (double)P.part_rows));
  int lo = (int)fmin(fmax(least, ceil(W / res)), 0x3fffffff);
  if (U < res) {
    // W / C + U parts at most: some C up to W / (res - U) fits
    int hi = max(lo, (int)fmin(ceil(W / (res - U)), 0x3fffffff));
    while (lo < hi) {
      const int C = (lo + hi) / 2;
      if (sum([C](const ChunkWork& w) { return (double)min((long long)w.units * chunk_parts(w.nk, C), 1ll << 20); }) <= res) hi = C;
      else lo = C + 1;
    }
  }
  return lo;
}

// sum over the wave by data-parallel moves: an inclusive sum within rows of 16, then
// the rows' last lanes
__device__ __forceinline__ double wave_total(double v) {
#define CHUNK_DPP_ADD(ctrl, rows)                                                                     \
  {                                                                                                   \
    const long long b = __double_as_longlong(v);                                                      \
    const int lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, ctrl, rows, 0xf, false);          \
    const int hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), ctrl, rows, 0xf, false);  \
    v += __longlong_as_double((long long)((uint64_t)(uint32_t)lo | (uint64_t)(uint32_t)hi << 32));    \
  }
  CHUNK_DPP_ADD(0x111, 0xf)
  CHUNK_DPP_ADD(0x112, 0xf)
  CHUNK_DPP_ADD(0x114, 0xf)
  CHUNK_DPP_ADD(0x118, 0xf)
  CHUNK_DPP_ADD(0x142, 0xa)
  CHUNK_DPP_ADD(0x143, 0xc)
#undef CHUNK_DPP_ADD
  const long long b = __double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, 63), hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63);
  return __longlong_as_double((long long)((uint64_t)lo | (uint64_t)hi << 32));
}

// sum over the workgroup's 1024 threads of v, and the sum before this thread (s: 16 values of LDS)
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

// One workgroup: divides the work of any number of sequences and clears the job queues.
// head[0] = jobs, head[1] = whether a tile is divided, head[8 + x] = the next job of
// XCD x's share.
__global__ void __launch_bounds__(1024) chunk_plan_kernel(ChunkArgs P, int keys_per_tile, int least_tiles, int res) {
  __shared__ long long s[16];
  constexpr int MAX_PER = CHUNK_MAX_SEQS / 1024;
  const int tid = threadIdx.x, per = (P.b + 1023) / 1024;
  ChunkWork w[MAX_PER];
#pragma unroll
  for (int u = 0; u < MAX_PER; ++u) {
    const int i = tid * per + u;
    w[u] = u < per && i < P.b ? chunk_work(P, chunk_seq(P, i), keys_per_tile) : ChunkWork{0, 0, 0};
  }
  const int C = chunk_part_length(P, least_tiles, res, [&](auto f) {
    double v = 0.0;
#pragma unroll
    for (int u = 0; u < MAX_PER; ++u) v += f(w[u]);
    long long total;
    (void)scan1024((long long)fmin(v, 0x1p52), s, total);  // (whole numbers; offsets that break the rules may give more)
    return (double)total;
  });
  long long jobs = 0, prows = 0;
#pragma unroll
  for (int u = 0; u < MAX_PER; ++u) {
    const long long parts = chunk_parts(w[u].nk, C);
    jobs += w[u].units * parts;
    if (parts > 1) prows += w[u].units * parts * w[u].prow;
  }
  long long njobs, nrows;
  long long j0 = scan1024(jobs, s, njobs), r0 = scan1024(prows, s, nrows);
#pragma unroll
  for (int u = 0; u < MAX_PER; ++u) {
    const int i = tid * per + u;
    if (u >= per || i >= P.b) continue;
    const long long parts = chunk_parts(w[u].nk, C);
    P.job_base[i] = (int)j0;
    P.seq_parts[i] = make_int2((int)parts, (int)r0);
    j0 += w[u].units * parts;
    if (parts > 1) r0 += w[u].units * parts * w[u].prow;
  }
  // sequences that do not overlap have at most 2^24 jobs or so: overlapping ones past 31
  // bits of them are not done
  if (njobs > INT32_MAX) njobs = nrows = 0;
  if (tid == 0) {
    P.head[0] = (int)njobs;
    P.head[1] = nrows > 0;
  }
  if (tid < ATTN_XCDS) P.head[8 + tid] = (int)(njobs * tid / ATTN_XCDS);
}

// The same division of at most 64 sequences by one wave, a lane a sequence: the job of
// workgroup `block` (seq -1: none), its job within the sequence and its parts.
struct ChunkJob {
  int seq, rel;
  int2 sp;
};
__device__ __forceinline__ ChunkJob chunk_wave_plan(const ChunkArgs& P, int keys_per_tile, int least_tiles, int res, int block) {
  const int lane = threadIdx.x & 63;
  const ChunkWork w = lane < P.b ? chunk_work(P, chunk_seq(P, lane), keys_per_tile) : ChunkWork{0, 0, 0};
  const int C = chunk_part_length(P, least_tiles, res, [&](auto f) { return wave_total(f(w)); });
  const int parts = chunk_parts(w.nk, C);
  const int jobs = w.units * parts, prows = parts > 1 ? jobs * w.prow : 0;
  int j = jobs, r = prows;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int a = __shfl_up(j, o, 64), b = __shfl_up(r, o, 64);
    if (lane >= o) {
      j += a;
      r += b;
    }
  }
  const int njobs = __shfl(j, 63, 64);
  if (block == 0) {  // for the merge
    if (lane < P.b) P.seq_parts[lane] = make_int2(parts, r - prows);
    const int any = __shfl(r, 63, 64);
    if (lane == 0) P.head[1] = any > 0;
  }
  const int x = block % ATTN_XCDS, job = (int)((long long)njobs * x / ATTN_XCDS) + block / ATTN_XCDS;
  ChunkJob out = {-1, 0, make_int2(1, 0)};
  if (job >= (int)((long long)njobs * (x + 1) / ATTN_XCDS)) return out;
  const unsigned long long past = __builtin_amdgcn_ballot_w64(j > job);
  out.seq = __builtin_ctzll(past);
  out.rel = job - __shfl(j - jobs, out.seq, 64);
  out.sp = make_int2(__shfl(parts, out.seq, 64), __shfl(r - prows, out.seq, 64));
  return out;
}

// The pages of a sequence, as a wave holds them: lane l has the block-table entry of the
// tile's key l (`load`; looked at only a tile later, because a look would wait for all
// loads in flight), its page (-1: no such key, or unmapped), and then the byte offset of
// that key's row of kv head g in the pools (page 0 for keys without one).
template <typename T, int DH>
struct ChunkPages {
  const ChunkArgs& P;
  const int32_t* row;  // the sequence's block-table row
  int g, keys, lane;
  static constexpr int KEYS = ChunkTile<T>::KEYS, RB = DH * (int)sizeof(T);
  __device__ __forceinline__ int load(int kt) const {
    return row[min((kt * KEYS + (lane & (KEYS - 1))) >> P.ps_shift, P.max_pages - 1)];
  }
  __device__ __forceinline__ int page(int kt, int entry) const {
    return kt * KEYS + (lane & (KEYS - 1)) < keys && entry >= 0 && entry < P.num_pages ? entry : -1;
  }
  __device__ __forceinline__ uint64_t offset(int kt, int page) const {
    const uint32_t stride = ((uint32_t)P.Hkv << P.ps_shift) * RB;  // bytes of a page
    const uint32_t at = ((uint32_t)g << P.ps_shift) + ((kt * KEYS + (lane & (KEYS - 1))) & ((1 << P.ps_shift) - 1));
    return (uint64_t)(uint32_t)max(page, 0) * stride + at * RB;
  }
  static __device__ __forceinline__ unsigned long long mapped(int page) {
    return __builtin_amdgcn_ballot_w64(page >= 0) & (KEYS == 64 ? ~0ull : (1ull << KEYS) - 1);
  }
};

// 16 bytes a lane from `at` past `rows` and the constant `from`, to LDS at d + from
template <int from, typename Rows>
__device__ __forceinline__ void chunk_copy_piece(const Rows& rows, chunk_lds_t* d, uint32_t at) {
#if defined(__HIP_DEVICE_COMPILE__)  // (the host's pass does not know 16-byte pieces)
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, d, 16, at, 0, from, 0);
#endif
}

// A buffer of n bytes, `off` past `pool` (0x27000: plain 32-bit elements, no swizzle)
__device__ __forceinline__ auto chunk_rows(const void* pool, uint64_t off, int n) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)((uint64_t)pool + off), 0, n, 0x27000);
}

// Copies a tile's rows from `pool` straight to LDS (256 threads), given the keys' row
// offsets.  A wave copies KEYS / 4 consecutive rows, NL pieces of 1 KB in both places:
// where the rows share a page, one scalar address serves them all (the instruction's
// offset moves both sides) and the lanes' own offsets are those of every tile, so that
// the copy takes next to nothing of either unit; in smaller pages each piece has its
// own.  Those are buffer loads: while loads from the lanes' own addresses are in flight,
// the compiler lets every LDS read wait for all LDS reads before it.  Pages smaller than
// a piece's rows need such loads, which are waited for here for that reason.
template <typename T, int DH>
__device__ __forceinline__ void chunk_copy(const ChunkArgs& P, const void* pool, unsigned char* dst, uint64_t off, int wave,
                                           int lane) {
  constexpr int KEYS = ChunkTile<T>::KEYS, RB = DH * (int)sizeof(T), CH = RB / 16, NL = KEYS * CH / 256, RW = 64 / CH;
  static_assert(NL == 2 || NL == 4, "pieces");
  const int lo = (int)(uint32_t)off, hi = (int)(uint32_t)(off >> 32);
  asm volatile("" : "+v"(lane));  // (formed anew per tile: kept, the offsets would spill)
  chunk_lds_t* const d = (chunk_lds_t*)(dst + wave * NL * 1024);
  const int r0 = wave * (KEYS / 4);
  if ((1 << P.ps_shift) >= RW) {
    // (the swizzle permutes bits of the row, and the pieces' first rows share none with lane / CH)
    const uint32_t first = lane / CH * RB + (((lane % CH) ^ chunk_swz<T, DH>(lane / CH) ^ chunk_swz<T, DH>(r0)) << 4);
    auto at = [&](int i) { return first ^ (chunk_swz<T, DH>(i * RW) << 4); };
    auto lane_offset = [&](int r) {
      return (uint64_t)(uint32_t)__builtin_amdgcn_readlane(lo, r) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, r) << 32;
    };
    if ((1 << P.ps_shift) >= KEYS / 4) {
      const auto rows = chunk_rows(pool, lane_offset(r0), NL * 1024);
      chunk_copy_piece<0>(rows, d, at(0));
      chunk_copy_piece<1024>(rows, d, at(1));
      if constexpr (NL > 2) {
        chunk_copy_piece<2 * 1024>(rows, d, at(2));
        chunk_copy_piece<3 * 1024>(rows, d, at(3));
      }
    } else {
#pragma unroll
      for (int i = 0; i < NL; ++i)
        chunk_copy_piece<0>(chunk_rows(pool, lane_offset(r0 + i * RW), 1024), (chunk_lds_t*)(dst + (wave * NL + i) * 1024), at(i));
    }
  } else {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int r = (wave * NL + i) * RW + lane / CH, c = (lane % CH) ^ chunk_swz<T, DH>(r);
      const uint64_t at = (uint64_t)(uint32_t)__shfl(lo, r, 64) | (uint64_t)(uint32_t)__shfl(hi, r, 64) << 32;
      __builtin_amdgcn_global_load_lds((const void*)((const char*)pool + at + c * 16),
                                       (chunk_lds_t*)(dst + (wave * NL + i) * 1024), 16, 0, 0);
    }
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
  }
}

// The row that a lane works for: query row `lane % 32` of its wave's block of 32 (both
// halves of the wave share them).
struct ChunkRow {
  bool valid;
  int t, q;      // position (-1: no row, and it attends nothing), row of the tile
  size_t at;     // (row, head) in Q, O and the LSE
};
__device__ __forceinline__ ChunkRow chunk_row(const ChunkArgs& P, const ChunkSeq& S, int tile, int g, int wave, int lane) {
  const int G = P.H / P.Hkv, QPT = CHUNK_ROWS / G;
  ChunkRow r;
  r.q = wave * 32 + (lane & 31);
  const int pl = r.q / G;
  r.valid = pl < QPT && tile * QPT + pl < S.m;
  r.t = r.valid ? S.base + tile * QPT + pl : -1;
  r.at = ((size_t)S.r0 + tile * QPT + pl) * P.H + g * G + (r.q - pl * G);
  return r;
}

// Which keys of which unit a workgroup attends.
struct ChunkSpan {
  int t0, tlo, tend;  // position of the tile's first row; key tiles
};
__device__ __forceinline__ ChunkSpan chunk_span(const ChunkArgs& P, const ChunkSeq& S, int tile, int part, int parts, int keys) {
  const int QPT = CHUNK_ROWS / (P.H / P.Hkv);
  const int t_hi = S.base + min(tile * QPT + QPT, S.m) - 1;
  const int nkt = (min(max(t_hi + 1, 0), S.keys) + keys - 1) / keys;
  const int per = (nkt + parts - 1) / parts;
  return {S.base + tile * QPT, part * per, min(part * per + per, nkt)};
}

// A product with P = 0 would turn an infinite or NaN value of a key that a row does not
// attend into NaN.  In tiles with such keys, values of keys without a page (not in vm)
// are zeroed; infinite and NaN elements of the others are added to the rows that do
// attend them (the sum is not finite whatever their weight) and then zeroed too.
template <typename T, int DH>
__device__ __forceinline__ void chunk_fix_values(unsigned char* vb, unsigned long long* bad_keys, int k0,
                                                 unsigned long long vm, int t, floatx16_t* o, int wave, int lane) {
  constexpr int RB = DH * (int)sizeof(T), CH = RB / 16, NL = ChunkTile<T>::KEYS * CH / 256;
  asm volatile("" : "+v"(lane));  // (nothing of this rare path is kept outside it)
  if (threadIdx.x == 0) *bad_keys = 0;
  lds_barrier();
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    asm volatile("" ::: "memory");  // (few loads at a time: registers are short)
    const int r = ((wave * NL + i) * 64 + lane) / CH;
    uint4* pv = (uint4*)(vb + (wave * NL + i) * 1024 + lane * 16);
    if (!((vm >> r) & 1)) {
      *pv = make_uint4(0, 0, 0, 0);
    } else {
      const uint4 u = *pv;
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
      bool bad = false;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        bad = bad || (w[e] & 0x7f800000u) == 0x7f800000u || (sizeof(T) == 2 && (w[e] & 0x7f80u) == 0x7f80u);
      if (bad) atomicOr(bad_keys, 1ull << r);
    }
  }
  lds_barrier();
  unsigned long long bm = uniform64(*bad_keys);
  if (!bm) return;
  for (; bm; bm &= bm - 1) {
    const int r = __builtin_ctzll(bm);
    const bool on = k0 + r <= t;
#pragma unroll
    for (int dv = 0; dv < DH / 2; ++dv) {
      // dimension 32 dt + 8 (v / 4) + 4 lk + v % 4: its 16-byte chunk, and the place in it
      const int dt = dv / 16, v = dv % 16, lk = lane >> 5 & 1;
      const int c = sizeof(T) == 2 ? dt * 4 + (v >> 2) : dt * 8 + 2 * (v >> 2) + lk;
      if (dv % 4 == 0) asm volatile("" ::: "memory");
      const T* x = (const T*)(vb + r * RB + ((c ^ chunk_swz<T, DH>(r)) << 4)) + (sizeof(T) == 2 ? 4 * lk : 0) + (v & 3);
      const float f = Act<T>::to_f32(*x);
      o[dt][v] += on && !(fabsf(f) < INFINITY) ? f : 0.f;
    }
  }
  lds_barrier();
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    asm volatile("" ::: "memory");
    T* pv = (T*)(vb + (wave * NL + i) * 1024 + lane * 16);
#pragma unroll
    for (int e = 0; e < 16 / (int)sizeof(T); ++e)
      if (!(fabsf(Act<T>::to_f32(pv[e])) < INFINITY)) pv[e] = 0;
  }
  lds_barrier();
}

// A row's result, or its unnormalized sums and (max, sum) where the unit is in parts.
template <typename T, int DH>
__device__ __forceinline__ void chunk_store(const ChunkArgs& P, const ChunkSeq& S, int tile, int g, int rel, int2 sp,
                                            const floatx16_t* o, float m_run, float l_run, int wave, int lane) {
  asm volatile("" : "+v"(lane));  // (the row is formed anew: kept through the loop, it would spill)
  const ChunkRow R = chunk_row(P, S, tile, g, wave, lane);
  const int lk = lane >> 5;
  if (!R.valid) return;
  if (sp.x > 1) {
    const int G = P.H / P.Hkv;
    const size_t row = (size_t)sp.y + (size_t)rel * (min(S.m, CHUNK_ROWS / G) * G) + R.q;
    float* po = P.part_o + row * DH;
#pragma unroll
    for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4)
        *(float4*)(po + dt * 32 + 8 * v4 + 4 * lk) =
            make_float4(o[dt][4 * v4 + 0], o[dt][4 * v4 + 1], o[dt][4 * v4 + 2], o[dt][4 * v4 + 3]);
    if (lk == 0) *(float2*)(P.part_ml + row * 2) = make_float2(m_run, l_run);
    return;
  }
  const float inv_l = l_run == 0.f ? 0.f : 1.0f / l_run;
  T* op = (T*)P.O + R.at * DH;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int v4 = 0; v4 < 4; ++v4) {
      const int d0 = dt * 32 + 8 * v4 + 4 * lk;
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = l_run == 0.f ? 0.f : o[dt][4 * v4 + e] * inv_l;
      if constexpr (sizeof(T) == 2) *(uint2*)(op + d0) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
      else *(float4*)(op + d0) = make_float4(x[0], x[1], x[2], x[3]);
    }
  if (P.lse && lk == 0) P.lse[R.at] = l_run == 0.f ? -INFINITY : (m_run + log2f(l_run)) * LN2;
}

// The transposing LDS read of 8 bytes.  Without the qualifier the compiler would let each
// wait for every direct-to-LDS load in flight, the next tiles' among them; what a tile
// reads has been waited for at its barrier.
__device__ __forceinline__ uint2 chunk_read_tr(lds_s16x4_t* __restrict p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(p));
}

// One job: a tile's rows over one part of its keys, two tiles of keys in LDS by turns, one
// barrier a tile.  Bound by the keys' bytes where rows are few: one row over 131000 cached
// (32/32 heads of 128, 2.1 GB) 363 us, 5.9 TB/s; 32 sequences of 5 new tokens over up to
// 16000 (28/4 heads, 280 MB) 55 us, 5.1 TB/s, of which 4.7 us pass before the first key.
template <typename T, int DH>
__device__ __forceinline__ void chunk_job(const ChunkArgs& P, const int seq, const int rel, const int2 sp) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int KEYS = ChunkTile<T>::KEYS, NST = KEYS / 32;
  constexpr int RB = DH * (int)sizeof(T);       // bytes of a row
  constexpr int TB = KEYS * RB;                 // bytes of a tile
  // two buffers of K and V (4 TB bytes; dynamic, because the compiler makes every read
  // of a static array wait for the direct-to-LDS loads in flight)
  extern __shared__ __align__(256) unsigned char tiles[];
  __shared__ unsigned long long bad_s;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lk = lane >> 5;
  const ChunkSeq S = chunk_seq(P, seq);
  const int ntile = (S.m + CHUNK_ROWS / (P.H / P.Hkv) - 1) / (CHUNK_ROWS / (P.H / P.Hkv));
  const int part = rel % sp.x, tile = ntile - 1 - (rel / sp.x) % ntile, g = rel / sp.x / ntile;
  const ChunkRow R = chunk_row(P, S, tile, g, wave, lane);
  const ChunkSpan span = chunk_span(P, S, tile, part, sp.x, KEYS);
  const int t = R.t, t0 = span.t0, tend = span.tend;
  const bool wave_live = __builtin_amdgcn_ballot_w64(R.valid) != 0;

  // Q^T as the B operand of S^T = K Q^T.  bf16: lane supplies dimensions
  // 16 ks + 8 lk + 0..7; fp32: 8 ks + 4 lk + e for step (ks, e)
  constexpr int NQ = BF ? DH / 16 : DH / 8;
  uint4 qb[NQ];
  {
    const T* qp = (const T*)P.Q + R.at * DH;
#pragma unroll
    for (int ks = 0; ks < NQ; ++ks)
      qb[ks] = R.valid ? *(const uint4*)(qp + (BF ? ks * 16 + lk * 8 : ks * 8 + lk * 4)) : make_uint4(0, 0, 0, 0);
  }

  floatx16_t o[DH / 32];
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[dt][v] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const float qk_scale = P.sm_scale * LOG2E;

  const ChunkPages<T, DH> pages = {P, P.table + (size_t)seq * P.max_pages, g, S.keys, lane};
  auto load_tile = [&](int kt, int pg, int buf) {
    const uint64_t off = pages.offset(kt, pg);
    chunk_copy<T, DH>(P, P.k_pages, tiles + buf * 2 * TB, off, wave, lane);
    chunk_copy<T, DH>(P, P.v_pages, tiles + buf * 2 * TB + TB, off, wave, lane);
  };
  constexpr unsigned long long ALL = KEYS == 64 ? ~0ull : 0xffffffffull;

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

  int kt = span.tlo, buf = 0;
  int pg = -1;
  unsigned long long vcur = 0;
  if (kt < tend) {
    pg = pages.page(kt, pages.load(kt));
    load_tile(kt, pg, 0);
    vcur = pages.mapped(pg);
    pg = pages.load(kt + 1);
  }
  for (; kt < tend; ++kt, buf ^= 1) {
    // this wave's loads of the tile are done; after the barrier everyone's are,
    // and every wave is done with the other buffer
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const int k0 = kt * KEYS;
    unsigned char* const tb = tiles + buf * 2 * TB;
    asm volatile("" : "+v"(o_row), "+v"(o_tr[0]), "+v"(o_tr[1]));  // (formed anew per tile: kept, they would spill)
    const int pn = pages.page(kt + 1, pg);
    const unsigned long long vnext = pages.mapped(pn);
    if (kt + 1 < tend) {
      load_tile(kt + 1, pn, buf ^ 1);
      pg = pages.load(kt + 2);
    }
    const bool diag = k0 + KEYS - 1 > t0, gaps = vcur != ALL;
    if (diag || gaps) chunk_fix_values<T, DH>(tb + TB, &bad_s, k0, vcur, t, o, wave, lane);
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
        // P goes to the matrix unit as two bf16 numbers, the upper half of the weight less 2^-20
        // of it and the rest (together within 2^-16 of the weight), so that a token here is as
        // exact as in the decode step.  The rest is positive: 0, or less behind a half rounded
        // up, would turn an infinite value into NaN.  The calls of this loop are bound by the
        // keys' bytes, and the second product mostly hides behind them: 366 -> 369 us for one
        // row over 131000 cached, 64.5 -> 65.8 for 32 sequences of 5.
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          const int st = ks >> 1, v0 = 8 * (ks & 1);
          uint32_t hi4[4], lo4[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float a = s[st][v0 + 2 * j], b = s[st][v0 + 2 * j + 1];
            const uint32_t a1 = __float_as_uint(fmaf(a, -0x1p-20f, a)), b1 = __float_as_uint(fmaf(b, -0x1p-20f, b));
            hi4[j] = __builtin_amdgcn_perm(b1, a1, 0x07060302u);  // both upper halves
            lo4[j] = pack_bf16x2(a - __uint_as_float(a1 & 0xffff0000u), b - __uint_as_float(b1 & 0xffff0000u));
          }
          const uint4 pu = make_uint4(hi4[0], hi4[1], hi4[2], hi4[3]), pr = make_uint4(lo4[0], lo4[1], lo4[2], lo4[3]);
          uint4 vu[DH / 32];
#pragma unroll
          for (int dt = 0; dt < DH / 32; ++dt) {
            const uint2 lo = chunk_read_tr((lds_s16x4_t*)(tb + TB + (o_tr[0] ^ (dt << 6)) + ks * 16 * RB));
            const uint2 hi = chunk_read_tr((lds_s16x4_t*)(tb + TB + (o_tr[1] ^ (dt << 6)) + ks * 16 * RB));
            vu[dt] = make_uint4(lo.x, lo.y, hi.x, hi.y);
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8_t*)&vu[dt], *(const bf16x8_t*)&pu, o[dt], 0, 0, 0);
          }
#pragma unroll
          for (int dt = 0; dt < DH / 32; ++dt)
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8_t*)&vu[dt], *(const bf16x8_t*)&pr, o[dt], 0, 0, 0);
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

  chunk_store<T, DH>(P, S, tile, g, rel, sp, o, m_run, l_run, wave, lane);
}

// LDS read of 16 bytes at a 32-bit address
__device__ __forceinline__ bf16x8_t lds_read16(uint32_t a) {
  return *(const __attribute__((address_space(3))) bf16x8_t*)(uintptr_t)a;
}

// the larger of x in lanes l and l ^ 32
__device__ __forceinline__ float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// The same job (bf16, pages of 16 keys or more), pipelined inside the wave for calls that
// the matrix unit bounds: 32 keys at a time, the matrix unit forms the scores of the next
// tile while the vector unit takes this tile's exponentials and sums, then the products
// with the values; none waits for the other.  K runs a tile ahead of V in LDS: an
// iteration reads K(t + 1) and V(t) and loads K(t + 2) and V(t + 1), with one barrier.
// 2048 tokens over 30005 cached, 28/4 heads of 128: 0.90 ms (1.01 PFLOP/s, 0.885 to 0.923
// from card to card; the plain loop before its second product 0.961 ms, a large product
// reaches 1.4 PFLOP/s); 2304 tokens, whose tiles fill every workgroup, 1.08 PFLOP/s.  What
// bounds it: matrix and vector cycles add up (busy in 50% and 40% of all cycles, with 56 of
// 512 places empty) at a clock of 1.9 GHz of 2.4 (1.8 in a loop of nothing but products).
// Removing waits alone, 2% of the cycles, took no time off; removing vector instructions
// did: page lookups in scalar registers (15% of them) 2%, no maxima but where the reference
// moves 6%.  Not kept: 64 keys at a time (181 spilled registers, 3.1 ms), 64 rows a wave
// with the fragments shared (340).
template <int DH>
__device__ __forceinline__ void chunk_job_piped(const ChunkArgs& P, const int seq, const int rel, const int2 sp) {
  using T = bf16_t;
  constexpr int KEYS = 64, RB = DH * 2, TB = KEYS * RB;
  // K buffers at 0 and TB, V buffers at 2 TB and 3 TB
  extern __shared__ __align__(256) unsigned char tiles[];
  __shared__ unsigned long long bad_s;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lr = lane & 31, lk = lane >> 5;
  const ChunkSeq S = chunk_seq(P, seq);
  const int ntile = (S.m + CHUNK_ROWS / (P.H / P.Hkv) - 1) / (CHUNK_ROWS / (P.H / P.Hkv));
  const int part = rel % sp.x, tile = ntile - 1 - (rel / sp.x) % ntile, g = rel / sp.x / ntile;
  const ChunkRow R = chunk_row(P, S, tile, g, wave, lane);
  const ChunkSpan span = chunk_span(P, S, tile, part, sp.x, KEYS);
  const int t = R.t, t0 = span.t0, tlo = span.tlo, tend = span.tend;

  uint4 qb[DH / 16];
#pragma unroll
  for (int ks = 0; ks < DH / 16; ++ks)
    qb[ks] = R.valid ? *(const uint4*)((const T*)P.Q + R.at * DH + ks * 16 + lk * 8) : make_uint4(0, 0, 0, 0);

  floatx16_t o[DH / 32];
  float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[dt][v] = 0.f;
  const float qk_scale = P.sm_scale * LOG2E;

  // Pages: lane j of every four has the block-table entry of the tile's j-th 16 keys (a
  // page has at least as many), looked at a tile later, because a look waits for all loads
  // in flight; the rest is scalar.  A wave copies 16 keys' rows, in pieces of 1 KB.
  constexpr int NL = RB / 64, CH = RB / 16, RW = 64 / CH;
  const int32_t* const table = P.table + (size_t)seq * P.max_pages;
  const int key0 = (lane & 3) * 16;
  auto entries = [&](int kt) { return table[min((kt * KEYS + key0) >> P.ps_shift, P.max_pages - 1)]; };
  struct Pages {
    unsigned long long vm;  // keys with a page
    uint64_t off;           // offset of this wave's first row in the pools (in page 0 without one)
  };
  auto look = [&](int kt, int entry) {
    const bool ok = entry >= 0 && entry < P.num_pages && kt * KEYS + key0 < S.keys;
    const uint32_t m4 = (uint32_t)__builtin_amdgcn_ballot_w64(ok);
    const uint32_t page = m4 >> wave & 1 ? (uint32_t)__builtin_amdgcn_readlane(entry, wave) : 0;
    const uint32_t in = ((uint32_t)g << P.ps_shift) + ((kt * KEYS + wave * 16) & ((1 << P.ps_shift) - 1));
    const int left = S.keys - kt * KEYS;
    Pages r = {~0ull, (uint64_t)page * (((uint32_t)P.Hkv << P.ps_shift) * RB) + in * RB};
    if ((m4 & 15) != 15 || left < KEYS) {
      r.vm = 0;
      for (int j = 0; j < 4; ++j) r.vm |= m4 >> j & 1 ? 0xffffull << (16 * j) : 0;
      if (left < KEYS) r.vm &= (1ull << max(left, 0)) - 1;
    }
    return r;
  };
  uint32_t at[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i)
    at[i] = lane / CH * RB + (((lane % CH) ^ chunk_swz<T, DH>(wave * 16 + i * RW + lane / CH)) << 4);
  auto copy = [&](const void* pool, unsigned char* dst, uint64_t off) __attribute__((always_inline)) {
    const auto rows = chunk_rows(pool, off, NL * 1024);
    chunk_lds_t* const d = (chunk_lds_t*)(dst + wave * NL * 1024);
    chunk_copy_piece<0>(rows, d, at[0]);
    chunk_copy_piece<1024>(rows, d, at[1]);
    if constexpr (NL > 2) {
      chunk_copy_piece<2 * 1024>(rows, d, at[2]);
      chunk_copy_piece<3 * 1024>(rows, d, at[3]);
    }
  };
  auto load_k = [&](int kt, uint64_t off) { copy(P.k_pages, tiles + ((kt - tlo) & 1) * TB, off); };
  auto load_v = [&](int kt, uint64_t off) { copy(P.v_pages, tiles + (2 + ((kt - tlo) & 1)) * TB, off); };
  auto tile_barrier = [] { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

  const uint32_t lds0 = (uint32_t)(uintptr_t)(chunk_lds_t*)tiles;  // aligned to a row
  const uint32_t o_row = lds0 + lr * RB + ((lk ^ chunk_swz<T, DH>(lr)) << 4);
  uint32_t o_tr[2];
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    const int r = 4 * lk + 8 * hf + ((lane & 15) >> 2);
    o_tr[hf] = lds0 + r * RB + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ chunk_swz<T, DH>(r)) << 4) + (lane & 1) * 8;
  }

  // S = K Q^T of half st of the tile in the K buffer at kb
  auto product = [&](floatx16_t& s, uint32_t kb, int st) __attribute__((always_inline)) {
    const floatx16_t z = {};
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks) {
      const bf16x8_t k = lds_read16((o_row ^ (ks << 5)) + kb + st * 32 * RB);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, *(const bf16x8_t*)&qb[ks], ks ? s : z, 0, 0, 0);
    }
  };
  // masks of a tile that reaches past the first row's position, or has keys without a page
  auto mask = [&](floatx16_t& s, int kt, int st, unsigned long long vm) {
    int lk4 = 4 * lk;
    asm volatile("" : "+v"(lk4));
    vm >>= lk4;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int j = st * 32 + 8 * (v >> 2) + (v & 3);
      if (kt * KEYS + j + lk4 > t || !((vm >> j) & 1)) s[v] = -INFINITY;
    }
  };
  // The reference of the exponentials.  Any that they do not all underflow against gives the
  // same sums, so it is looked at only where a lane's 16 weights add up to more than `limit`:
  // one of them then exceeds 2^8, and the reference moves to the row's maximum.  A row that
  // has none yet is looked at whatever the sum (0 may be underflow), one that attends nothing
  // never for being empty.
  float limit = t < 0 ? 4096.f : -1.f;
  auto reference = [&](const floatx16_t& s) __attribute__((always_inline)) {
    float mx = s[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
    mx = pair_max(mx * qk_scale);  // (the scale is positive)
    if (mx > m_run + 8.f) {
      // (nothing is summed yet where m_run is -inf)
      const float alpha = m_run == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - mx);
      m_run = mx;
      limit = 4096.f;
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[dt][v] *= alpha;
    }
  };
  unsigned long long vm = 0, vm1 = 0;  // keys of tiles kt and kt + 1 with a page
  uint64_t off1 = 0;                   // where tile kt + 1 is
  int e2 = -1;                         // block-table entries of tile kt + 2
  auto special = [&](int kt, unsigned long long v) { return kt * KEYS + KEYS - 1 > t0 || v != ~0ull; };
  if (tlo < tend) {
    floatx16_t s0, s1, u0, u1;  // (a tile's halves, by turns)
    {
      const int e0 = entries(tlo), e1 = entries(tlo + 1);
      const Pages p0 = look(tlo, e0), p1 = look(tlo + 1, e1);
      load_k(tlo, p0.off);
      load_v(tlo, p0.off);
      if (tlo + 1 < tend) load_k(tlo + 1, p1.off);
      e2 = entries(tlo + 2);
      vm = p0.vm;
      vm1 = p1.vm;
      off1 = p1.off;
    }
    tile_barrier();
    // both halves of K(tlo) are read before the first iteration's loads replace it
    product(s0, 0, 0);
    product(s1, 0, 1);
    if (special(tlo, vm)) mask(s0, tlo, 0, vm);
    reference(s0);
    // tile kt, of scores s0 and s1; leaves those of the next in n0 and n1
    // (odd: the tile lies in the odd buffers, counted from tlo)
    auto tile = [&](int kt, floatx16_t& s0, floatx16_t& s1, floatx16_t& n0, floatx16_t& n1, auto odd_t) __attribute__((always_inline)) {
      constexpr int odd = decltype(odd_t)::value;
      tile_barrier();  // K(kt + 1) and V(kt) are there; K(kt) and V(kt - 1) are free
      const Pages p2 = look(kt + 2, e2);
      if (kt + 1 < tend) load_v(kt + 1, off1);
      if (kt + 2 < tend) load_k(kt + 2, p2.off);
      off1 = p2.off;
      e2 = entries(kt + 3);
      const bool masked = special(kt, vm), masked1 = special(kt + 1, vm1);
      if (masked) chunk_fix_values<T, DH>(tiles + (2 + odd) * TB, &bad_s, kt * KEYS, vm, t, o, wave, lane);
      constexpr uint32_t kb = (odd ^ 1) * TB, vb = (2 + odd) * TB;
      // Half st of the tile, of scores s; leaves the next tile's in n: their products
      // between this half's exponentials and sums, then its products with the values.  One
      // product takes the matrix unit 32 cycles, more than a step's vector instructions take
      // the other; the steps are pinned, because the compiler groups each kind of instruction.
      auto half = [&](const floatx16_t& s, floatx16_t& n, int st) __attribute__((always_inline)) {
        constexpr int NK = DH / 16, ND = DH / 32, PER = 16 / NK;  // steps, groups of dimensions, weights a step
        uint32_t pk[8];
        uint4 f0[ND], f1[ND];
        bf16x8_t kf[NK];
        float p[16], r2[2] = {0.f, 0.f};
        float bias = m_run == -INFINITY ? 0.f : -m_run;
        auto read_k = [&](int ks) { kf[ks] = lds_read16((o_row ^ (ks << 5)) + kb + st * 32 * RB); };
        auto read_v = [&](uint4* f, int dt, int ks) {
          const uint2 lo = chunk_read_tr((lds_s16x4_t*)(uintptr_t)((o_tr[0] ^ (dt << 6)) + vb + (2 * st + ks) * 16 * RB));
          const uint2 hi = chunk_read_tr((lds_s16x4_t*)(uintptr_t)((o_tr[1] ^ (dt << 6)) + vb + (2 * st + ks) * 16 * RB));
          f[dt] = make_uint4(lo.x, lo.y, hi.x, hi.y);
        };
        // P is rounded to bf16 for the matrix instruction (2^-8 of a weight, averaged over the
        // keys; the whole-prompt attention does the same), the sum keeps the fp32 weights: a
        // second product with the rest, as in the plain loop, takes 2048 over 30005 from 0.907
        // to 1.254 ms
        auto finish = [&](int u) {
#pragma unroll
          for (int v = u * PER; v < (u + 1) * PER; v += 2) {
            r2[0] += p[v];
            r2[1] += p[v + 1];
            pk[v / 2] = pack_bf16x2(p[v], p[v + 1]);
          }
        };
        read_k(0);
        read_k(1);
        read_k(2);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < NK; ++u) {
          if (u + 3 < NK) read_k(u + 3);
          else if (u + 3 - NK < ND) read_v(f0, u + 3 - NK, 0);
          const floatx16_t z = {};
          n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[u], *(const bf16x8_t*)&qb[u], u ? n : z, 0, 0, 0);
#pragma unroll
          for (int v = u * PER; v < (u + 1) * PER; ++v)
            p[v] = __builtin_amdgcn_exp2f(fmaf(s[v], qk_scale, bias));
          if (u > 0) finish(u - 1);
          __builtin_amdgcn_sched_barrier(0);
        }
        finish(NK - 1);
#pragma unroll
        for (int dt = 3; dt < ND; ++dt) read_v(f0, dt, 0);
        __builtin_amdgcn_sched_barrier(0);
        if (__builtin_amdgcn_ballot_w64(!(r2[0] + r2[1] <= limit)) != 0) {
          reference(s);
          bias = m_run == -INFINITY ? 0.f : -m_run;
          r2[0] = r2[1] = 0.f;
#pragma unroll
          for (int v = 0; v < 16; ++v) p[v] = __builtin_amdgcn_exp2f(fmaf(s[v], qk_scale, bias));
#pragma unroll
          for (int u = 0; u < NK; ++u) finish(u);
        }
        l_run += r2[0] + r2[1];  // this lane's keys
#pragma unroll
        for (int u = 0; u < 2 * ND; ++u) {
          const int dt = u % ND, v0 = 4 * (u / ND);
          if (u < ND) read_v(f1, u, 1);
          const uint4 pu = make_uint4(pk[v0], pk[v0 + 1], pk[v0 + 2], pk[v0 + 3]);
          const uint4& f = u < ND ? f0[dt] : f1[dt];
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8_t*)&f, *(const bf16x8_t*)&pu, o[dt], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      half(s0, n0, 0);
      if (masked) mask(s1, kt, 1, vm);
      half(s1, n1, 1);
      if (masked1) mask(n0, kt + 1, 0, vm1);
      vm = vm1;
      vm1 = p2.vm;
    };
    for (int kt = tlo;;) {
      tile(kt, s0, s1, u0, u1, std::integral_constant<int, 0>{});
      if (++kt >= tend) break;
      tile(kt, u0, u1, s0, s1, std::integral_constant<int, 1>{});
      if (++kt >= tend) break;
    }
  }
  l_run += __shfl_xor(l_run, 32, 64);
  chunk_store<T, DH>(P, S, tile, g, rel, sp, o, m_run, l_run, wave, lane);
}

// INLINE (at most 64 sequences, fewer (tile, head) pairs than the grid): the job of
// this workgroup by its own division.  Otherwise the division of chunk_plan_kernel:
// one job a workgroup where they fit the grid, else jobs from the XCD's queue, then
// from the next XCDs', until all eight are drained.
template <typename T, int DH, bool INLINE, bool PIPED>
__global__ void __launch_bounds__(256, 2) chunk_attn_kernel(ChunkArgs P, int res) {
  __shared__ ChunkJob job_s;
  const int lane = threadIdx.x & 63;
  if constexpr (INLINE) {
    if (threadIdx.x < 64) {
      const ChunkJob j = chunk_wave_plan(P, ChunkTile<T>::KEYS, ChunkTile<T>::LEAST, res, blockIdx.x);
      if (lane == 0) job_s = j;
    }
  }
  const int njobs = INLINE ? 0 : P.head[0];
  const bool queue = njobs > (int)gridDim.x;
  for (bool first = true;; first = false) {
    if (!first) {
      if (!queue) break;
      __syncthreads();  // every thread has finished the previous job and read job_s
    }
    if (!INLINE && threadIdx.x < 64) {
      int job = -1;
      if (!queue) {
        const int x = blockIdx.x % ATTN_XCDS;
        job = (int)((long long)njobs * x / ATTN_XCDS) + blockIdx.x / ATTN_XCDS;
        if (job >= (int)((long long)njobs * (x + 1) / ATTN_XCDS)) job = -1;
      } else {
        for (;;) {
          // the first XCD from this one on whose queue has not been seen empty
          const int x = (blockIdx.x + lane) % ATTN_XCDS;
          const int end = (int)((long long)njobs * (x + 1) / ATTN_XCDS);
          const int at = lane < ATTN_XCDS ? __hip_atomic_load(&P.head[8 + x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
          const unsigned long long some = __builtin_amdgcn_ballot_w64(lane < ATTN_XCDS && at < end);
          if (!some) break;
          const int l = __builtin_ctzll(some);
          int j = 0;
          if (lane == l) j = atomicAdd(&P.head[8 + x], 1);
          j = __shfl(j, l, 64);
          if (j < __shfl(end, l, 64)) {
            job = j;
            break;
          }
        }
      }
      ChunkJob r = {-1, 0, make_int2(1, 0)};
      if (job >= 0) {
        r.seq = wave_find(P.job_base, P.b, job, lane);
        r.rel = job - P.job_base[r.seq];
        r.sp = P.seq_parts[r.seq];
      }
      if (lane == 0) job_s = r;
    }
    __syncthreads();
    const ChunkJob r = job_s;
    if (r.seq < 0) break;
    const int seq = __builtin_amdgcn_readfirstlane(r.seq), rel = __builtin_amdgcn_readfirstlane(r.rel);
    const int2 sp = make_int2(__builtin_amdgcn_readfirstlane(r.sp.x), __builtin_amdgcn_readfirstlane(r.sp.y));
    if constexpr (PIPED) chunk_job_piped<DH>(P, seq, rel, sp);
    else chunk_job<T, DH>(P, seq, rel, sp);
    if (INLINE) break;
  }
}

// Merge of divided tiles: a wave per (row, head), its lanes 64 / C8 parts at a time x
// 8 dimensions each.  Bound by its two rounds of loads: 160 rows of 28 heads 6.0 us (6.5
// with four rounds).
template <typename T, int DH>
__global__ void __launch_bounds__(256) chunk_combine_kernel(ChunkArgs P) {
  constexpr int C8 = DH / 8, PG = 64 / C8;
  const int lane = threadIdx.x & 63, c8 = lane % C8, pg = lane / C8;
  const int G = P.H / P.Hkv, QPT = CHUNK_ROWS / G;
  // up to 64 sequences: each in a lane, loaded together (one wait instead of four)
  const bool few = P.b <= 64;
  const int li = min(lane, P.b - 1);
  const int start = P.row_start[li], end = P.row_start[few ? li + 1 : P.b];
  const int2 parts = P.seq_parts[li];
  const int first = __builtin_amdgcn_readlane(start, 0);
  const int last = min(few ? __builtin_amdgcn_readlane(end, P.b - 1) : __builtin_amdgcn_readfirstlane(end), P.rows);
  if (P.head[1] == 0) return;
  for (long long it = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); it < (long long)P.rows * P.H;
       it += (long long)gridDim.x * 4) {
    const int r = (int)(it / P.H), h = (int)(it % P.H), g = h / G;
    if (r < first || r >= last) continue;
    int2 sp;
    int r0, r1;
    if (few) {
      const int i = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(lane < P.b && start <= r));
      sp = make_int2(__builtin_amdgcn_readlane(parts.x, i), __builtin_amdgcn_readlane(parts.y, i));
      r0 = __builtin_amdgcn_readlane(start, i);
      r1 = __builtin_amdgcn_readlane(end, i);
    } else {
      const int i = __builtin_amdgcn_readfirstlane(wave_find(P.row_start, P.b, r, lane));
      sp = P.seq_parts[i];
      r0 = P.row_start[i];
      r1 = P.row_start[i + 1];
    }
    if (sp.x <= 1) continue;
    r0 = min(max(r0, 0), P.rows);  // (as chunk_seq)
    const int m = min(max(r1, r0), P.rows) - r0, j = r - r0;
    if (j >= m) continue;
    const int ntile = (m + QPT - 1) / QPT, tile = j / QPT, pl = j - tile * QPT;
    const int R = min(m, QPT) * G;  // rows of a part
    const size_t s0 = (size_t)sp.y + (size_t)(g * ntile + (ntile - 1 - tile)) * sp.x * R + pl * G + (h - g * G);
    const float2* ml = (const float2*)P.part_ml + s0;
    float mx = -INFINITY;
    for (int p = lane; p < sp.x; p += 64) mx = fmaxf(mx, ml[(size_t)p * R].x);
    mx = wave_max(mx);
    const float mu = mx == -INFINITY ? 0.f : mx;
    float l = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const float* po = P.part_o + s0 * DH + c8 * 8;
    for (int p = pg; p < sp.x; p += PG) {
      const float2 q = ml[(size_t)p * R];
      const float4 a = *(const float4*)(po + (size_t)p * R * DH);
      const float4 b = *(const float4*)(po + (size_t)p * R * DH + 4);
      if (q.y == 0.f) continue;  // nothing attended in this part
      const float w = __builtin_amdgcn_exp2f(q.x - mu);
      l += q.y * w;
      acc[0] += a.x * w;
      acc[1] += a.y * w;
      acc[2] += a.z * w;
      acc[3] += a.w * w;
      acc[4] += b.x * w;
      acc[5] += b.y * w;
      acc[6] += b.z * w;
      acc[7] += b.w * w;
    }
#pragma unroll
    for (int o = C8; o < 64; o <<= 1) {
      l += __shfl_xor(l, o, 64);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += __shfl_xor(acc[e], o, 64);
    }
    if (pg != 0) continue;
    const float inv_l = l == 0.f ? 0.f : 1.0f / l;
    T* op = (T*)P.O + ((size_t)r * P.H + h) * DH + c8 * 8;
    if constexpr (sizeof(T) == 2) {
      *(uint4*)op = make_uint4(pack_bf16x2(acc[0] * inv_l, acc[1] * inv_l), pack_bf16x2(acc[2] * inv_l, acc[3] * inv_l),
                               pack_bf16x2(acc[4] * inv_l, acc[5] * inv_l), pack_bf16x2(acc[6] * inv_l, acc[7] * inv_l));
    } else {
      *(float4*)op = make_float4(acc[0] * inv_l, acc[1] * inv_l, acc[2] * inv_l, acc[3] * inv_l);
      *(float4*)(op + 4) = make_float4(acc[4] * inv_l, acc[5] * inv_l, acc[6] * inv_l, acc[7] * inv_l);
    }
    if (P.lse && c8 == 0) P.lse[(size_t)r * P.H + h] = l == 0.f ? -INFINITY : (mu + log2f(l)) * LN2;
  }
}

// The kernels of a type and head dimension, allowed their two tile buffers of LDS on
// the current device, and the workgroups of them that it holds (a multiple of the
// XCDs; 0 when the runtime cannot tell), asked once a device.
struct ChunkKernels {
  void (*queued)(ChunkArgs, int);
  void (*inl)(ChunkArgs, int);
  void (*combine)(ChunkArgs);
  int res;
};
template <typename T, int DH, bool PIPED>
static ChunkKernels chunk_kernels() {
  static std::atomic<int> known[64];  // workgroups of each device, 0: not asked yet
  ChunkKernels k = {chunk_attn_kernel<T, DH, false, PIPED>, chunk_attn_kernel<T, DH, true, PIPED>,
                    chunk_combine_kernel<T, DH>, 0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return k;
  k.res = known[dev].load();
  if (k.res) return k;
  const size_t lds = (size_t)512 * DH;
  for (auto f : {k.queued, k.inl})
    if (hipFuncSetAttribute((const void*)f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) return k;
  k.res = std::min(resident_workgroups(k.queued, 256, lds), resident_workgroups(k.inl, 256, lds)) / ATTN_XCDS * ATTN_XCDS;
  known[dev].store(k.res);
  return k;
}

hipError_t launch_chunk_attention(int dtype, const ChunkArgs& a, hipStream_t s) {
  const int G = a.H / a.Hkv;
  const int keys = dtype == SAS_BF16 ? ChunkTile<bf16_t>::KEYS : ChunkTile<float>::KEYS;
  const int least = dtype == SAS_BF16 ? ChunkTile<bf16_t>::LEAST : ChunkTile<float>::LEAST;
  // the pipelined kernel where the average sequence fills more than half a tile: with fewer
  // rows the keys' bytes bound the call, and the plain loop's second product hides behind
  // them.  By it and by the plain loop, us: 32 sequences over 4000 cached, 28/4 heads, of 5
  // tokens 64.7 and 65.3, of 9 (63 rows) 69.3 and 67.3, of 10 (70 rows) 70.9 and 74.0, of 18
  // 79.3 and 85.4; 8 over 2000, 32/32 heads, of 1 62.3 and 61.3, of 64 76.0 and 75.9, of 65
  // 76.4 and 78.0, of 128 106 and 113
  const bool piped = dtype == SAS_BF16 && a.ps_shift >= 4 && (long long)a.rows * G > (long long)CHUNK_ROWS / 2 * std::min(a.b, a.rows);
  // (tile, kv head) pairs, at most
  const long long tiles = ((long long)a.rows / (CHUNK_ROWS / G) + std::min(a.b, a.rows)) * a.Hkv;
  ChunkKernels k;
  if (dtype != SAS_BF16) k = a.dh == 128 ? chunk_kernels<float, 128, false>() : chunk_kernels<float, 64, false>();
  else if (piped) k = a.dh == 128 ? chunk_kernels<bf16_t, 128, true>() : chunk_kernels<bf16_t, 64, true>();
  else k = a.dh == 128 ? chunk_kernels<bf16_t, 128, false>() : chunk_kernels<bf16_t, 64, false>();
  const int res = k.res;
  if (res <= 0) return hipErrorInvalidValue;
  // the most jobs that there can be: tiles in parts of the least length
  const long long max_keys = (long long)a.max_pages << a.ps_shift;
  const long long part_keys = (long long)keys * least;
  const long long parts = a.part_rows > 0 ? (max_keys + part_keys - 1) / part_keys : 1;
  const long long most = (std::min<long long>(res, tiles * std::min<long long>(parts, res)) + ATTN_XCDS - 1) / ATTN_XCDS * ATTN_XCDS;
  const bool inl = a.b <= 64 && tiles < res;
  if (!inl) chunk_plan_kernel<<<1, 1024, 0, s>>>(a, keys, least, res);
  (inl ? k.inl : k.queued)<<<(unsigned)most, 256, 512 * a.dh, s>>>(a, res);
  if (parts > 1) {
    const long long waves = (long long)a.rows * a.H;
    k.combine<<<(unsigned)std::min<long long>((waves + 3) / 4, 8192), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace sas
