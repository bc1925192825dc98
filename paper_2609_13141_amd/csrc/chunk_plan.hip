// Pages and rows of a chunk of new tokens: block-table entries, slots and
// positions from the requests' lengths.
//
// Two prefix sums over the sequences (rows, pages wanted) decide everything;
// every workgroup forms them itself in LDS (12 bytes a sequence, from L2) and
// then takes its share of the rows, of the table entries to write and of the
// per-sequence outputs, so one launch does it.  A row finds its sequence by a
// binary search in LDS.
#include "common.h"
#include "kernels.h"

namespace sas {

constexpr int PLAN_NT = 256, PLAN_ROWS = 4;  // threads; consecutive rows of a thread

struct PlanSeq {
  int ctx, m, held, need;
};
__device__ __forceinline__ PlanSeq plan_seq(const PlanArgs& P, int i) {
  PlanSeq q;
  q.ctx = max(P.ctx_len[i], 0);
  q.m = max(P.new_len[i], 0);
  q.held = min(max(P.held[i], 0), P.max_pages);
  const long long end = ((long long)q.ctx + q.m + (1 << P.ps_shift) - 1) >> P.ps_shift;
  q.need = q.m > 0 ? max((int)min(end, (long long)P.max_pages) - q.held, 0) : 0;
  return q;
}

// largest i in [0, b) with start[i] <= x (start[0] <= x)
template <typename I>
__device__ __forceinline__ int find_start(const I* start, int b, I x) {
  int lo = 0, hi = b;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(PLAN_NT) plan_chunk_kernel(PlanArgs P) {
  extern __shared__ __align__(16) unsigned char plan_lds[];
  long long* const page0 = (long long*)plan_lds;        // [b + 1] pages wanted before sequence i
  int* const row0 = (int*)(page0 + P.b + 1);            // [b + 1] rows before sequence i
  __shared__ long long wsum[2][PLAN_NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (P.b + PLAN_NT - 1) / PLAN_NT;
  const int i0 = min(tid * per, P.b), i1 = min(i0 + per, P.b);
  long long nr = 0, np = 0;
  for (int i = i0; i < i1; ++i) {
    const PlanSeq q = plan_seq(P, i);
    nr += q.m;
    np += q.need;
  }
  long long xr = nr, xp = np;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long yr = __shfl_up(xr, o, 64), yp = __shfl_up(xp, o, 64);
    if (lane >= o) {
      xr += yr;
      xp += yp;
    }
  }
  if (lane == 63) {
    wsum[0][wave] = xr;
    wsum[1][wave] = xp;
  }
  __syncthreads();
  long long r = xr - nr, p = xp - np, all_r = 0, all_p = 0;
#pragma unroll
  for (int w = 0; w < PLAN_NT / 64; ++w) {
    if (w < wave) {
      r += wsum[0][w];
      p += wsum[1][w];
    }
    all_r += wsum[0][w];
    all_p += wsum[1][w];
  }
  for (int i = i0; i < i1; ++i) {
    const PlanSeq q = plan_seq(P, i);
    row0[i] = (int)min(r, (long long)P.rows);
    page0[i] = p;
    r += q.m;
    p += q.need;
  }
  const int total = (int)min(all_r, (long long)P.rows);
  if (tid == 0) {
    row0[P.b] = total;
    page0[P.b] = all_p;
  }
  __syncthreads();

  const int avail = min(max(P.free_count[0], 0), P.free_capacity);
  const int gtid = blockIdx.x * PLAN_NT + tid, nthreads = gridDim.x * PLAN_NT;
  // per-sequence outputs
  for (int i = gtid; i <= P.b; i += nthreads) {
    P.row_start[i] = row0[i];
    if (i == P.b) {
      P.free_out[0] = (int)(avail - min(all_p, (long long)avail));
      P.missing[0] = (int)min(max(all_p - avail, 0ll), 0x7fffffffll);
      break;
    }
    const PlanSeq q = plan_seq(P, i);
    // (tokens without a row are not in the chunk: attention places a sequence's rows from its end)
    P.kv_len[i] = (int)min((long long)q.ctx + (row0[i + 1] - row0[i]), 0x7fffffffll);
    P.held_out[i] = q.held + (int)min((long long)q.need, max(avail - page0[i], 0ll));
  }
  // table entries of the pages wanted, off the top of the stack in the sequences' order
  for (long long e = gtid; e < all_p; e += nthreads) {
    const int i = find_start(page0, P.b, e);
    const int held = min(max(P.held[i], 0), P.max_pages);
    P.table[(size_t)i * P.max_pages + held + (int)(e - page0[i])] = e < avail ? P.free_pages[avail - 1 - e] : -1;
  }
  // rows
  const int psm = (1 << P.ps_shift) - 1;
  for (long long base = (long long)gtid * PLAN_ROWS; base < P.rows; base += (long long)nthreads * PLAN_ROWS) {
    int oseq[PLAN_ROWS], opos[PLAN_ROWS];
    long long oslot[PLAN_ROWS];
    int i = base < total ? find_start(row0, P.b, (int)base) : P.b;
    int next = i < P.b ? row0[i + 1] : 0x7fffffff;
    PlanSeq q = {0, 0, 0, 0};
    if (i < P.b) q = plan_seq(P, i);
#pragma unroll
    for (int u = 0; u < PLAN_ROWS; ++u) {
      const long long x = base + u;
      oseq[u] = -1;
      opos[u] = -1;
      oslot[u] = -1;
      if (x >= total) continue;
      if (x >= next) {
        do ++i;
        while (row0[i + 1] <= x);
        next = row0[i + 1];
        q = plan_seq(P, i);
      }
      const long long at = (long long)q.ctx + (x - row0[i]);
      const long long pi = at >> P.ps_shift;
      int page = -1;
      if (pi < P.max_pages) {
        if (pi < q.held) {
          page = P.table[(size_t)i * P.max_pages + pi];
        } else {
          const long long e = page0[i] + (pi - q.held);
          if (e < avail) page = P.free_pages[avail - 1 - e];
        }
      }
      oseq[u] = i;
      opos[u] = (int)min(at, 0x7fffffffll);
      if (page >= 0 && page < P.num_pages) oslot[u] = ((long long)page << P.ps_shift) + (at & psm);
    }
    if (base + PLAN_ROWS <= P.rows) {
      *(int4*)(P.seq + base) = make_int4(oseq[0], oseq[1], oseq[2], oseq[3]);
      *(int4*)(P.pos + base) = make_int4(opos[0], opos[1], opos[2], opos[3]);
      *(longlong2*)(P.slot + base) = make_longlong2(oslot[0], oslot[1]);
      *(longlong2*)(P.slot + base + 2) = make_longlong2(oslot[2], oslot[3]);
    } else {
#pragma unroll
      for (int u = 0; u < PLAN_ROWS; ++u)
        if (base + u < P.rows) {
          P.seq[base + u] = oseq[u];
          P.pos[base + u] = opos[u];
          P.slot[base + u] = oslot[u];
        }
    }
  }
}

hipError_t launch_plan_chunk(const PlanArgs& a, hipStream_t s) {
  const size_t lds = (size_t)(a.b + 1) * 12;
  const int grid = std::max(1, std::min(1024, cdiv(a.rows, PLAN_NT * PLAN_ROWS)));
  plan_chunk_kernel<<<grid, PLAN_NT, lds, s>>>(a);
  return hipGetLastError();
}

}  // namespace sas
