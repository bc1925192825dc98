// Verification of drafted tokens against the target's probabilities.
//
// Sequence i drafted m tokens x_0 .. x_{m-1}; they are accepted in order while
// u_j q_j(x_j) < p_j(x_j).  One more token is drawn by the inverse CDF of the
// sequence's uniform u: from max(p - q, 0) at the first token that was not
// accepted (from p without x_j when the draft has no probabilities; from p
// itself when nothing is left), from p after the last when all were.
//
// Only one row of p and one of q are read in full, b vocab (4 or 8) bytes.  The
// vocabulary is cut in sixteen, the sixteenth that the uniform falls into in sixteen
// again, until a wave can scan it token by token (eight a lane, loaded together; 64 at a
// time 2.4 us more of 29, all waves scanning another 1).  A workgroup a sequence does it
// all; for large vocabularies sixteen take a sequence's sums first (verify_one).
// Products, differences and sums are fp64: products of the fp32 inputs are exact there,
// differences and sums are rounded, so that a token's border in the CDF is uncertain by a
// few 1e-16 of the sum (an fp32 sum's by 1e-7).  The forms add in different orders: a
// uniform that close to a border may draw either neighbour, by the number of sequences.
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace sas {

constexpr int VERIFY_WAVES = 16;  // and pieces of a cut
constexpr int VERIFY_LANE = 8;    // tokens that a lane loads together

// tokens of a piece of n, whole steps of a wave
__host__ __device__ __forceinline__ int verify_piece(int n) { return ((n + VERIFY_WAVES - 1) / VERIFY_WAVES + 63) / 64 * 64; }

// The rows that sequence i's last token is drawn from, found by every wave.
struct VerifyRow {
  int r0, acc;      // first drafted token, accepted ones
  const float* p;   // target row
  const float* q;   // draft row, or null
  int skip;         // token that is left out (a draft without probabilities), or -1
};
__device__ __forceinline__ VerifyRow verify_row(const VerifyArgs& P, int i) {
  const int lane = threadIdx.x & 63;
  const int r0 = min(max(P.start[i], 0), P.rows);
  const int m = min(min(max(P.start[i + 1], r0), P.rows) - r0, P.max_draft);
  // 64 drafted tokens at a time; the first that is not accepted ends the search
  int acc = m;
  for (int j0 = 0; j0 < m; j0 += 64) {
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

__device__ __forceinline__ double wave_sum_f64(double x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// sum of the weights of tokens [a, b) (negative and NaN ones count as zero), a lane every 64th
__device__ __forceinline__ double verify_sum(const VerifyRow& v, int a, int b) {
  double w[4] = {0.0, 0.0, 0.0, 0.0};
  int e = a + (threadIdx.x & 63);
  // the loads of 8 tokens together, also of the last ones (those past the end load the last
  // token, without weight; a batch of 2 where that is enough): one at a time, pieces of less
  // than 512 tokens made the kernel before slower than the one workgroup (8 x 100003: 21.5
  // -> 14.4 us)
  auto batch = [&](auto with_q, auto width, int last) __attribute__((always_inline)) {
    constexpr int N = decltype(width)::value;
    float p[N], q[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int x = min(e + u * 64, last);
      p[u] = v.p[x];
      q[u] = 0.f;
      if constexpr (decltype(with_q)::value) q[u] = v.q[x];
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const double d = (double)p[u] - (double)q[u];
      w[u & 3] += e + u * 64 <= last && e + u * 64 != v.skip && d > 0.0 ? d : 0.0;
    }
    e += N * 64;
  };
  auto all = [&](auto with_q) __attribute__((always_inline)) {
    const std::integral_constant<int, 8> eight;
    while (e + 7 * 64 < b) batch(with_q, eight, 0x7fffffff);
    if (e + 2 * 64 < b) batch(with_q, eight, b - 1);
    else if (e < b) batch(with_q, std::integral_constant<int, 2>(), b - 1);
  };
  if (v.q) all(std::true_type());
  else all(std::false_type());
  return wave_sum_f64((w[0] + w[1]) + (w[2] + w[3]));
}

// Sums of the sixteen pieces of [e0, e1), `len` tokens each, into s.
__device__ __forceinline__ void verify_sums(const VerifyRow& v, int e0, int e1, int len, double* s) {
  const int wave = threadIdx.x >> 6;
  const int a = (int)min((long long)e0 + (long long)wave * len, (long long)e1);
  const double sum = verify_sum(v, a, (int)min((long long)a + len, (long long)e1));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[wave] = sum;
  __syncthreads();
}

// part[i][k][j]: the sum of piece j of piece k; workgroup (k, i), a wave four of them
__global__ void __launch_bounds__(256) verify_sum_kernel(VerifyArgs P) {
  const int k = blockIdx.x, i = blockIdx.y, wave = threadIdx.x >> 6;
  const VerifyRow v = verify_row(P, i);
  const int len = verify_piece(P.vocab), sub = verify_piece(len);
  const int e0 = (int)min((long long)k * len, (long long)P.vocab), e1 = (int)min((long long)e0 + len, (long long)P.vocab);
  for (int j = wave * 4; j < wave * 4 + 4; ++j) {
    const int a = (int)min((long long)e0 + (long long)j * sub, (long long)e1);
    const double sum = verify_sum(v, a, (int)min((long long)a + sub, (long long)e1));
    if ((threadIdx.x & 63) == 0) P.part[((size_t)i * VERIFY_WAVES + k) * VERIFY_WAVES + j] = sum;
  }
}

// SUMS: verify_sum_kernel has taken the sums of the first two cuts
template <bool SUMS>
__global__ void __launch_bounds__(VERIFY_WAVES * 64) verify_kernel(VerifyArgs P) {
  __shared__ double s[VERIFY_WAVES], part[SUMS ? VERIFY_WAVES : 1][VERIFY_WAVES];
  const int i = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  if constexpr (SUMS) {
    if (tid < VERIFY_WAVES * VERIFY_WAVES)
      part[tid / VERIFY_WAVES][tid % VERIFY_WAVES] = P.part[(size_t)i * VERIFY_WAVES * VERIFY_WAVES + tid];
  }
  VerifyRow v = verify_row(P, i);
  int e0 = 0, e1 = P.vocab, len = verify_piece(P.vocab);
  if constexpr (SUMS) {
    __syncthreads();
    if (tid < VERIFY_WAVES) {
      double x = 0.0;
      for (int j = 0; j < VERIFY_WAVES; ++j) x += part[tid][j];
      s[tid] = x;
    }
    __syncthreads();
  } else {
    verify_sums(v, e0, e1, len, s);
  }
  double total = 0.0;
  for (int k = 0; k < VERIFY_WAVES; ++k) total += s[k];
  bool known = SUMS;  // part holds the sums of the next cut
  if (!(total > 0.0) && (v.q || v.skip >= 0)) {  // nothing left over: the target itself
    v.q = nullptr;
    v.skip = -1;
    known = false;
    verify_sums(v, e0, e1, len, s);
    for (int k = 0; k < VERIFY_WAVES; ++k) total += s[k];
  }
  const double aim = (double)P.u_sample[i] * total;
  // the piece that the aim falls into: the first whose end lies past it, or the last of
  // any weight (sums of other pieces may differ in their last bits)
  double before = 0.0;
  int token = -1;
  if (total > 0.0) {
    for (;;) {
      int pick = -1;
      double at = before, to = before;
      for (int k = 0; k < VERIFY_WAVES; ++k) {
        if (!(s[k] > 0.0)) continue;
        pick = k;
        at = to;
        to += s[k];
        if (to > aim) break;
      }
      if (pick < 0) break;  // (not reached: some piece has weight)
      before = at;
      e0 += pick * len;
      e1 = min(e0 + len, e1);
      if (e1 - e0 <= 64 * VERIFY_LANE) break;
      const int whole = len;
      len = verify_piece(known ? whole : e1 - e0);
      if (known) {
        __syncthreads();  // (every thread has read s)
        if (tid < VERIFY_WAVES) s[tid] = part[SUMS ? pick : 0][tid];
        __syncthreads();
        known = false;
      } else {
        verify_sums(v, e0, e1, len, s);
      }
    }
    if (tid >= 64) return;  // (the others have no more to do)
    // token by token, a lane eight of them
    const int b0 = e0 + lane * VERIFY_LANE;
    float p[VERIFY_LANE], q[VERIFY_LANE];
#pragma unroll
    for (int u = 0; u < VERIFY_LANE; ++u) p[u] = v.p[min(b0 + u, e1 - 1)];
#pragma unroll
    for (int u = 0; u < VERIFY_LANE; ++u) q[u] = 0.f;
    if (v.q) {
#pragma unroll
      for (int u = 0; u < VERIFY_LANE; ++u) q[u] = v.q[min(b0 + u, e1 - 1)];
    }
    double w[VERIFY_LANE], sum = 0.0;
#pragma unroll
    for (int u = 0; u < VERIFY_LANE; ++u) {
      const double d = (double)p[u] - (double)q[u];
      w[u] = b0 + u < e1 && b0 + u != v.skip && d > 0.0 ? d : 0.0;
      sum += w[u];
    }
    double x = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_up(x, o, 64);
      if (lane >= o) x += y;
    }
    double to = __shfl_up(x, 1, 64);  // the sum before this lane's tokens, and then of them
    to = lane ? before + to : before;
    int hit = -1, some = -1;  // the first token past the aim, the last of any weight
#pragma unroll
    for (int u = 0; u < VERIFY_LANE; ++u) {
      to += w[u];
      if (w[u] > 0.0) {
        some = b0 + u;
        if (hit < 0 && to > aim) hit = b0 + u;
      }
    }
    const unsigned long long hits = __builtin_amdgcn_ballot_w64(hit >= 0);
    const unsigned long long any = __builtin_amdgcn_ballot_w64(some >= 0);
    if (hits) token = __shfl(hit, __builtin_ctzll(hits), 64);
    else if (any) token = __shfl(some, 63 - __builtin_clzll(any), 64);
  }
  if (tid >= 64) return;
  const int W = P.max_draft + 1;
  for (int j = lane; j < W; j += 64)
    P.out[(size_t)i * W + j] = j < v.acc ? P.tokens[v.r0 + j] : j == v.acc ? token : -1;
  if (tid == 0) P.accepted[i] = v.acc;
}

hipError_t launch_verify_drafts(const VerifyArgs& a, hipStream_t s) {
  if (verify_one(a.b, a.vocab)) {
    verify_kernel<false><<<a.b, VERIFY_WAVES * 64, 0, s>>>(a);
  } else {
    verify_sum_kernel<<<dim3(VERIFY_WAVES, a.b), 256, 0, s>>>(a);
    verify_kernel<true><<<a.b, VERIFY_WAVES * 64, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace sas
