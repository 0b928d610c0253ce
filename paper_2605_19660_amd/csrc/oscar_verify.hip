// oscar_verify_drafts: which drafted tokens stand, and the token that follows them.
//
//   draft t stands      iff u_t q_t(x_t) < p_t(x_t)   (u < p / q without the division), and all before it do
//   a                   = drafts that stand; a = n (all of them) or the first that does not
//   weights of token a  = max(p_a - q_a, 0), or p_a where those are all zero; p_n for a = n
//   token a             = the smallest i with w_0 + ... + w_i > u_T (w_0 + ... + w_{V-1})
//
// Products and sums are in 64 bits: the comparison of two 24-bit factors with a 24-bit number is then
// exact, and the sums of a row differ between orders of summation by 1e-13 of its mass at most, so that
// the token does not depend on how the row is cut.
//
// What bounds it: one row of p and one of q a sequence are read, everything else is a few numbers.  The
// rows are cut into pieces of 4096 tokens so that few sequences still fill the chip: the first pass works
// out a (each workgroup for itself: three dependent loads) and sums its piece; the second finds the piece
// that holds the token from the sums, and in it the token, from a piece that is still in the L2.  Both scan
// in registers.  fp32, 64 sequences of 128003 tokens: 13.4 + 4.6 us, 4.9 TB/s in the first (a copy reaches
// 5.0); one of 32000: 5.0 + 3.7, latency.  In one launch, a workgroup of 16 waves a sequence, those take 44.6
// and 16.6 us: one CU's 64-bit arithmetic is what a long row then waits for.
#include "oscar_common.h"

namespace {

constexpr int PIECE = 4096;      // tokens of a workgroup's piece
constexpr int PER = PIECE / 256; // of a thread's part

struct VerifyParams {
  const void *p, *q;
  const int32_t *drafts, *draft_lens;
  const float* u;
  int32_t *n_new, *tokens;
  double2* sums;        // [batch][pieces]: sum of max(p - q, 0), sum of p
  int32_t* rows;        // [batch]: a
  int T, pieces;
  int64_t V;
};

// A probability: what is not above zero (NaN among it) counts as zero, infinity as the largest number.
template <typename E> __device__ __forceinline__ float probability(E e) {
  const float x = to_f32<E>(e);
  return x > 0.0f ? fminf(x, 3.402823466e38f) : 0.0f;
}

// Drafts of sequence b that stand, by the whole workgroup.
template <typename E> __device__ __forceinline__ int standing(const VerifyParams& P, int b, int* s_first) {
  const int n = P.draft_lens ? min(max(P.draft_lens[b], 0), P.T) : P.T;
  if (threadIdx.x == 0) *s_first = n;
  __syncthreads();
  for (int t = threadIdx.x; t < n; t += 256) {
    const int64_t x = P.drafts[(int64_t)b * P.T + t];
    bool ok = x >= 0 && x < P.V;
    if (ok) {
      const double pt = probability(reinterpret_cast<const E*>(P.p)[((int64_t)b * (P.T + 1) + t) * P.V + x]);
      const double qt = probability(reinterpret_cast<const E*>(P.q)[((int64_t)b * P.T + t) * P.V + x]);
      ok = (double)P.u[(int64_t)b * (P.T + 1) + t] * qt < pt;
    }
    if (!ok) {
      atomicMin(s_first, t);
      break;
    }
  }
  __syncthreads();
  return *s_first;
}

// The rows that decide the token behind a standing drafts (q: null where there is none to subtract).
template <typename E> struct Rows {
  const E *p, *q;
  __device__ __forceinline__ Rows(const VerifyParams& P, int b, int a, int n) {
    p = reinterpret_cast<const E*>(P.p) + ((int64_t)b * (P.T + 1) + a) * P.V;
    q = a < n ? reinterpret_cast<const E*>(P.q) + ((int64_t)b * P.T + a) * P.V : nullptr;
  }
};

// Up to N consecutive elements of a row (rows of odd lengths start anywhere: the loads carry no
// alignment beyond the element's).
template <typename E, int N> __device__ __forceinline__ void load_part(const E* row, int count, float* x) {
  if (count == N) {
    E e[N];
    __builtin_memcpy(e, row, sizeof(e));
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = probability(e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = i < count ? probability(row[i]) : 0.0f;
  }
}

__device__ __forceinline__ double weight(float p, float q) { return fmax((double)p - (double)q, 0.0); }

// The sum over the lanes up to this one, of a wave: four steps inside rows of 16 lanes, two that carry a row's last
// lane on (as lane permutations through LDS the six steps wait for it six times).
template <int CTRL, int ROWS> __device__ __forceinline__ double moved(double v) {
  const uint64_t bits = __double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(bits >> 32), CTRL, ROWS, 0xf, false);
  return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));   // 0 where no lane gives
}
__device__ __forceinline__ double wave_scan(double v) {
  v += moved<0x111, 0xf>(v);   // row_shr:1, 2, 4, 8
  v += moved<0x112, 0xf>(v);
  v += moved<0x114, 0xf>(v);
  v += moved<0x118, 0xf>(v);
  v += moved<0x142, 0xa>(v);   // row_bcast:15 into rows 1 and 3
  v += moved<0x143, 0xc>(v);   // row_bcast:31 into rows 2 and 3
  return v;
}
__device__ __forceinline__ double of_lane(double v, int lane) {   // lane: the same in all
  const uint64_t bits = __double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)bits, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(bits >> 32), lane);
  return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}

template <typename E> __global__ __launch_bounds__(256) void oscar_verify_sums_kernel(VerifyParams P) {
  __shared__ int s_first;
  __shared__ double2 s_wave[4];
  const int b = blockIdx.y, piece = blockIdx.x, tid = threadIdx.x;
  const int n = P.draft_lens ? min(max(P.draft_lens[b], 0), P.T) : P.T;
  const int a = standing<E>(P, b, &s_first);
  const Rows<E> rows(P, b, a, n);
  // vectors of 16 bytes side by side: the order of a sum does not matter here
  constexpr int VEC = 16 / sizeof(E);
  double r = 0.0, s = 0.0;
  float p[PER], q[PER] = {};
#pragma unroll
  for (int v = 0; v < PER / VEC; ++v) {
    const int64_t i = (int64_t)piece * PIECE + (v * 256 + tid) * VEC;
    const int count = (int)min(max(P.V - i, (int64_t)0), (int64_t)VEC);
    load_part<E, VEC>(rows.p + i, count, p + v * VEC);
    if (rows.q) load_part<E, VEC>(rows.q + i, count, q + v * VEC);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    r += weight(p[i], q[i]);
    s += p[i];
  }
  r = wave_scan(r);
  s = wave_scan(s);
  if (tid % 64 == 63) s_wave[tid / 64] = make_double2(r, s);
  __syncthreads();
  if (tid == 0) {
    P.sums[(int64_t)b * P.pieces + piece] = make_double2((s_wave[0].x + s_wave[1].x) + (s_wave[2].x + s_wave[3].x),
                                                        (s_wave[0].y + s_wave[1].y) + (s_wave[2].y + s_wave[3].y));
    if (piece == 0) P.rows[b] = a;
  }
}

template <typename E> __global__ __launch_bounds__(256) void oscar_verify_pick_kernel(VerifyParams P) {
  __shared__ double s_wave[4];
  __shared__ int s_hit, s_last;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = P.draft_lens ? min(max(P.draft_lens[b], 0), P.T) : P.T;
  const int a = P.rows[b];
  const float u = P.u[(int64_t)b * (P.T + 1) + P.T];
  const double2* sums = P.sums + (int64_t)b * P.pieces;
  if (tid == 0) s_hit = PIECE, s_last = -1;
  // Which weights, and their sum: every wave for itself, 64 pieces at a time.
  double sum_r = 0.0, sum_p = 0.0;
  for (int c0 = 0; c0 < P.pieces; c0 += 64) {
    const double2 w = c0 + lane < P.pieces ? sums[c0 + lane] : make_double2(0.0, 0.0);
    sum_r += of_lane(wave_scan(w.x), 63);
    sum_p += of_lane(wave_scan(w.y), 63);
  }
  const bool rest = sum_r > 0.0;
  const double target = (u > 0.0f ? (double)u : 0.0) * (rest ? sum_r : sum_p);
  // the first piece whose sums pass the target; if rounding lets none pass, the last with any weight
  int piece = -1, last_piece = -1;
  double base = 0.0, done = 0.0;
  for (int c0 = 0; c0 < P.pieces && piece < 0; c0 += 64) {
    const double2 both = c0 + lane < P.pieces ? sums[c0 + lane] : make_double2(0.0, 0.0);
    const double w = rest ? both.x : both.y, upto = wave_scan(w);
    const uint64_t some = __ballot(w > 0.0), past = __ballot(w > 0.0 && done + upto > target);
    if (some) last_piece = c0 + 63 - __builtin_clzll(some);
    if (past) {
      const int at = __builtin_ctzll(past);
      piece = c0 + at;
      base = at == 0 ? done : done + of_lane(upto, max(at - 1, 0));
    }
    done += of_lane(upto, 63);
  }
  const bool passed = piece >= 0;
  if (!passed) piece = last_piece;
  __syncthreads();
  if (piece >= 0) {   // (the same for all)
    const Rows<E> rows(P, b, a, n);
    const int64_t i0 = (int64_t)piece * PIECE + tid * PER;
    const int count = (int)min(max(P.V - i0, (int64_t)0), (int64_t)PER);
    float p[PER], q[PER] = {};
    load_part<E, PER>(rows.p + i0, count, p);
    if (rest && rows.q) load_part<E, PER>(rows.q + i0, count, q);
    double w[PER], part = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) part += w[i] = weight(p[i], q[i]);
    const double upto = wave_scan(part);
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    double cum = base;
#pragma unroll
    for (int v = 0; v < 3; ++v) cum += v < wave ? s_wave[v] : 0.0;
    cum += upto - part;
    int hit = PIECE, last = -1;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      cum += w[i];
      last = w[i] > 0.0 ? tid * PER + i : last;
      hit = hit == PIECE && w[i] > 0.0 && cum > target ? tid * PER + i : hit;
    }
    // the wave's first that passes and its last with any weight
    const uint64_t past = __ballot(hit < PIECE), some = __ballot(last >= 0);
    if (past && lane == __builtin_ctzll(past)) atomicMin(&s_hit, hit);
    if (some && lane == 63 - __builtin_clzll(some)) atomicMax(&s_last, last);
    __syncthreads();
  }
  const int token = piece < 0 ? 0 : piece * PIECE + (passed && s_hit < PIECE ? s_hit : s_last);
  int32_t* out = P.tokens + (int64_t)b * (P.T + 1);
  for (int t = tid; t <= P.T; t += 256)
    out[t] = t < a ? P.drafts[(int64_t)b * P.T + t] : t == a ? token : -1;
  if (tid == 0) P.n_new[b] = a + 1;
}

template <typename E> void launch(const VerifyParams& P, int batch, hipStream_t st) {
  hipLaunchKernelGGL((oscar_verify_sums_kernel<E>), dim3(P.pieces, batch), dim3(256), 0, st, P);
  hipLaunchKernelGGL((oscar_verify_pick_kernel<E>), dim3(batch), dim3(256), 0, st, P);
}

int pieces_of(int32_t vocab) { return (vocab + PIECE - 1) / PIECE; }

}  // namespace

extern "C" size_t oscar_verify_workspace_bytes(int32_t batch, int32_t vocab) {
  if (batch <= 0 || vocab <= 0 || vocab > OSCAR_VERIFY_MAX_VOCAB) return 0;
  return (size_t)batch * (pieces_of(vocab) * sizeof(double2) + sizeof(double));
}

extern "C" int oscar_verify_drafts(const void* target, const void* draft, const int32_t* drafts,
                                   const int32_t* draft_lens, const float* u, int32_t batch, int32_t T,
                                   int32_t vocab, int32_t dtype, int32_t* n_new, int32_t* tokens,
                                   void* workspace, size_t workspace_bytes, void* stream) {
  if (dtype != OSCAR_F32 && dtype != OSCAR_BF16 && dtype != OSCAR_F16) return OSCAR_ERR_INVALID_ARG;
  if (batch < 0 || batch > 65535 || T < 0 || T > OSCAR_VERIFY_MAX_DRAFTS || vocab < 1 || vocab > OSCAR_VERIFY_MAX_VOCAB)
    return OSCAR_ERR_INVALID_ARG;
  if (batch == 0) return OSCAR_OK;
  if (!target || !u || !n_new || !tokens || (T > 0 && (!draft || !drafts))) return OSCAR_ERR_INVALID_ARG;
  const size_t esize = dtype == OSCAR_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(target) % esize != 0 || reinterpret_cast<uintptr_t>(draft) % esize != 0)
    return OSCAR_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < oscar_verify_workspace_bytes(batch, vocab) ||
      (reinterpret_cast<uintptr_t>(workspace) & 15) != 0)
    return OSCAR_ERR_WORKSPACE;
  VerifyParams P = {};
  P.p = target;
  P.q = draft;
  P.drafts = drafts;
  P.draft_lens = draft_lens;
  P.u = u;
  P.n_new = n_new;
  P.tokens = tokens;
  P.T = T;
  P.V = vocab;
  P.pieces = pieces_of(vocab);
  P.sums = reinterpret_cast<double2*>(workspace);
  P.rows = reinterpret_cast<int32_t*>(P.sums + (size_t)batch * P.pieces);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (dtype == OSCAR_F32)
    launch<float>(P, batch, st);
  else if (dtype == OSCAR_BF16)
    launch<__hip_bfloat16>(P, batch, st);
  else
    launch<__half>(P, batch, st);
  if (hipGetLastError() != hipSuccess) return OSCAR_ERR_HIP;
  return OSCAR_OK;
}
