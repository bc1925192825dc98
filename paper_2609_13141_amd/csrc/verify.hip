// Verification of drafted tokens against the target's probabilities.
//
// Sequence i drafted m tokens x_0 .. x_{m-1}; they are accepted in order while
// u_j q_j(x_j) < p_j(x_j).  One more token is drawn by the inverse CDF of the
// sequence's uniform u: from max(p - q, 0) at the first token that was not
// accepted (from p without x_j when the draft has no probabilities; from p
// itself when nothing is left), from p after the last when all were.
//
// Only one row of p and one of q are read in full, b vocab (4 or 8) bytes:
// verify_sum_kernel cuts them into pieces, a workgroup each, and leaves the pieces'
// sums; verify_pick_kernel, a thread a piece, finds the one that the uniform falls
// into by a prefix sum and rescans that piece alone, each thread a run of it.  Differences and sums are fp64: the
// fp32 inputs' products and differences are exact there, and a token's border
// in the CDF is some 1e-16 wide rather than the 1e-7 of an fp32 sum.
#include "common.h"
#include "kernels.h"

namespace sas {

constexpr int VERIFY_NT = 256;

// The rows that sequence i's last token is drawn from, found by the first wave.
struct VerifyRow {
  int r0, acc;      // first drafted token, accepted ones
  const float* p;   // target row
  const float* q;   // draft row, or null
  int skip;         // token that is left out (a draft without probabilities), or -1
};
// `known`: the accepted tokens, or -1 to find them
__device__ __forceinline__ VerifyRow verify_row(const VerifyArgs& P, int i, int known) {
  const int lane = threadIdx.x & 63;
  const int r0 = min(max(P.start[i], 0), P.rows);
  const int m = min(min(max(P.start[i + 1], r0), P.rows) - r0, P.max_draft);
  // 64 drafted tokens at a time; the first that is not accepted ends the search
  int acc = known >= 0 ? known : m;
  for (int j0 = 0; known < 0 && j0 < m; j0 += 64) {
    const int j = j0 + lane;
    bool ok = true;
    if (j < m) {
      const int x = P.tokens[r0 + j];
      ok = false;
      if (x >= 0 && x < P.vocab) {
        const double px = P.target[(size_t)(r0 + i + j) * P.vocab + x];
        const double qx = P.draft ? P.draft[(size_t)(r0 + j) * P.vocab + x] : 1.0;
        ok = (double)P.u_accept[r0 + j] * qx < px;
      }
    }
    const unsigned long long no = __builtin_amdgcn_ballot_w64(!ok);
    if (no) {
      acc = j0 + __builtin_ctzll(no);
      break;
    }
  }
  VerifyRow v;
  v.r0 = r0;
  v.acc = acc;
  v.p = P.target + (size_t)(r0 + i + acc) * P.vocab;
  const bool stop = acc < m;
  v.q = stop && P.draft ? P.draft + (size_t)(r0 + acc) * P.vocab : nullptr;
  v.skip = stop && !P.draft ? P.tokens[r0 + acc] : -1;
  return v;
}

// weights of token e: (left over, target); negative and NaN values count as zero
__device__ __forceinline__ double verify_pos(double x) { return x > 0.0 ? x : 0.0; }
__device__ __forceinline__ double verify_left(const VerifyRow& v, int e, float p, float q) {
  return e == v.skip ? 0.0 : verify_pos((double)p - (double)q);
}

__device__ __forceinline__ double wave_sum_f64(double x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

__global__ void __launch_bounds__(VERIFY_NT) verify_sum_kernel(VerifyArgs P, int len) {
  __shared__ double red[2][VERIFY_NT / 64];
  const int i = blockIdx.y, piece = blockIdx.x;
  const VerifyRow v = verify_row(P, i, -1);
  if (piece == 0 && threadIdx.x == 0) P.accepted[i] = v.acc;
  const int e0 = piece * len, e1 = min(e0 + len, P.vocab);
  double left = 0.0, all = 0.0;
  for (int e = e0 + threadIdx.x; e < e1; e += VERIFY_NT) {
    const float p = v.p[e], q = v.q ? v.q[e] : 0.f;
    left += verify_left(v, e, p, q);
    all += verify_pos((double)p);
  }
  left = wave_sum_f64(left);
  all = wave_sum_f64(all);
  if ((threadIdx.x & 63) == 0) {
    red[0][threadIdx.x >> 6] = left;
    red[1][threadIdx.x >> 6] = all;
  }
  __syncthreads();
  if (threadIdx.x < 2) {
    double t = 0.0;
    for (int w = 0; w < VERIFY_NT / 64; ++w) t += red[threadIdx.x][w];
    P.part[((size_t)i * gridDim.x + piece) * 2 + threadIdx.x] = t;
  }
}

// sum before this thread of v over the workgroup, and the whole (s: 4 values of LDS)
__device__ __forceinline__ double scan_f64(double v, double* s, double& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) s[wave] = x;
  __syncthreads();
  double at = 0.0, sum = 0.0;
#pragma unroll
  for (int w = 0; w < VERIFY_NT / 64; ++w) {
    if (w < wave) at += s[w];
    sum += s[w];
  }
  total = sum;
  x = __shfl_up(x, 1, 64);
  return at + (lane ? x : 0.0);
}

__global__ void __launch_bounds__(VERIFY_NT) verify_pick_kernel(VerifyArgs P, int len, int pieces) {
  __shared__ double s[VERIFY_NT / 64];
  __shared__ int hit, some;  // the first piece or token past the uniform, the last of any weight
  __shared__ double base_s[VERIFY_NT];
  const int i = blockIdx.x, tid = threadIdx.x;
  const double* part = P.part + (size_t)i * pieces * 2;
  const double w0 = tid < pieces ? part[2 * tid] : 0.0, w1 = tid < pieces ? part[2 * tid + 1] : 0.0;
  VerifyRow v = verify_row(P, i, P.accepted[i]);
  if (tid == 0) {
    hit = 0x7fffffff;
    some = -1;
  }
  double left, all;
  const double b0 = scan_f64(w0, s, left), b1 = scan_f64(w1, s, all);
  if (!(left > 0.0)) {  // nothing left over: the target itself
    v.q = nullptr;
    v.skip = -1;
  }
  const double w = left > 0.0 ? w0 : w1, before = left > 0.0 ? b0 : b1;
  const double aim = (double)P.u_sample[i] * (left > 0.0 ? left : all);
  base_s[tid] = before;
  if (w > 0.0) {
    if (before + w > aim) atomicMin(&hit, tid);
    atomicMax(&some, tid);
  }
  __syncthreads();
  const int piece = hit != 0x7fffffff ? hit : some;
  __syncthreads();
  if (tid == 0) {
    hit = 0x7fffffff;
    some = -1;
  }
  if (piece >= 0) {
    // thread t's run of the piece: len / 256 tokens
    const int run = len / VERIFY_NT, e0 = piece * len + tid * run, e1 = min(e0 + run, P.vocab);
    double sum = 0.0, total;
    for (int e = e0; e < e1; ++e) sum += verify_left(v, e, v.p[e], v.q ? v.q[e] : 0.f);
    double at = base_s[piece] + scan_f64(sum, s, total);
    if (sum > 0.0) {
      int first = 0x7fffffff, last = -1;
      for (int e = e0; e < e1; ++e) {
        const double x = verify_left(v, e, v.p[e], v.q ? v.q[e] : 0.f);
        if (!(x > 0.0)) continue;
        at += x;
        if (first == 0x7fffffff && at > aim) first = e;
        last = e;
      }
      if (first != 0x7fffffff) atomicMin(&hit, first);
      atomicMax(&some, last);
    }
  }
  __syncthreads();
  const int W = P.max_draft + 1;
  for (int j = tid; j < W; j += VERIFY_NT) {
    int t = -1;
    if (j < v.acc) t = P.tokens[v.r0 + j];
    else if (j == v.acc) t = hit != 0x7fffffff ? hit : some;
    P.out[(size_t)i * W + j] = t;
  }
}

hipError_t launch_verify_drafts(const VerifyArgs& a, hipStream_t s) {
  // pieces of whole 256-token steps, at most a thread of the second kernel each: enough
  // workgroups to read the rows from the whole chip, and no more, since each looks the
  // accepted tokens up first
  const int steps = cdiv(a.vocab, VERIFY_NT), want = std::max(VERIFY_MIN_PIECES, std::min(VERIFY_PIECES, 2048 / a.b));
  const int len = cdiv(steps, std::min(steps, want)) * VERIFY_NT, pieces = cdiv(a.vocab, len);
  verify_sum_kernel<<<dim3(pieces, a.b), VERIFY_NT, 0, s>>>(a, len);
  verify_pick_kernel<<<a.b, VERIFY_NT, 0, s>>>(a, len, pieces);
  return hipGetLastError();
}

}  // namespace sas
