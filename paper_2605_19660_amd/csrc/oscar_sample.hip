// oscar_sample: a token from every row of logits, from given random numbers.
//
//   w_i = exp((l_i - max l) / temperature); in order of falling (l_i, -i):
//   the first top_k; of those the first whose weights reach top_p of their sum; of those the ones with w >= min_p
//   token = the smallest i with w_0 + .. + w_i > u * sum over what stays
//
// Every filter keeps a prefix of that order, so that what stays is everything from one pair (logit, index) on: the pair
// is held as one 64-bit number, (logit as an ordered integer, ~index), and the search is for that number, the cut.
// Weights are worked out in 64 bits.  Where many are added by atomics they count as multiples of 2^-(62 - log2 of
// the vocabulary): whole numbers, so that no order of additions changes a bit.
//
// A workgroup of 16 waves takes a row.
//  - top_k up to 1024: each thread knows the largest of its logits, and the k-th largest of the 1024 is no larger
//    than the k-th largest of all.  What lies above it (some more than k) goes to LDS and is sorted there.
//  - else the cut is searched by a histogram over the distance to the largest logit (equal steps, which spreads
//    a row over the bins, as the bits of the numbers would not); the bin that holds the cut goes to LDS and is sorted.
//    A bin that does not fit is split by the bits of its numbers until it does or holds one number only.
// What bounds it: the 64-bit exponentials of one CU where no top_k spares them, else latency.
#include "oscar_common.h"

namespace {

constexpr int THREADS = 1024, WAVES = 16;
constexpr int BINS = 1024;
constexpr int CAP = 4096;                  // numbers sorted in LDS
constexpr uint32_t DEAD = 0x007fffffu;     // key of -inf

struct SampleParams {
  const void* logits;
  int64_t stride;
  int V, fixed;        // vocabulary; binary places of a weight that is added by atomics
  const float *temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t* tokens;
  float* probs;
};

// Ordered integers: equal for equal numbers (both zeros are one), DEAD for -inf and NaN.
__device__ __forceinline__ uint32_t key_of(float x) {
  x = x == x ? fminf(x, 3.402823466e38f) + 0.0f : -INFINITY;
  const uint32_t b = __float_as_uint(x);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float number_of(uint32_t key) {
  return __uint_as_float(key ^ (key >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ uint64_t place_of(uint32_t key, int i) { return (uint64_t)key << 32 | (uint32_t)~i; }

template <typename T> __device__ __forceinline__ T shfl_up_any(T v, int d) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __shfl_up((uint32_t)bits, d), hi = __shfl_up((uint32_t)(bits >> 32), d);
  return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
}
template <typename T> __device__ __forceinline__ T wave_scan(T v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const T o = shfl_up_any(v, d);
    v += lane >= d ? o : T(0);
  }
  return v;
}
// Sum over the threads up to this one; all: over all.  s: WAVES numbers.
template <typename T> __device__ __forceinline__ T group_scan(T v, T* s, T* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_scan(v);
  __syncthreads();
  if (lane == 63) s[wave] = v;
  __syncthreads();
  T before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    before += w < wave ? s[w] : T(0);
    sum += s[w];
  }
  *all = sum;
  return v + before;
}
__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int d) {
  const uint32_t lo = __shfl_xor((uint32_t)v, d), hi = __shfl_xor((uint32_t)(v >> 32), d);
  return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t group_max(uint64_t v, uint64_t* s) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint64_t o = shfl_xor64(v, d);
    v = o > v ? o : v;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) v = s[w] > v ? s[w] : v;
  return v;
}

struct Shared {
  uint64_t list[CAP];
  uint64_t mass[BINS];
  uint32_t count[BINS];
  double part[BINS];         // sums of pieces of the row
  uint64_t wave64[WAVES];
  double wave_f[WAVES];
  uint32_t n;
  int found;
  uint64_t hit;
};

// Falling order of list[0 .. n), by the workgroup; returns with the list in place for all.
__device__ __forceinline__ void sort_list(uint64_t* list, int n) {
  int size = 2;
  while (size < n) size *= 2;
  for (int i = n + threadIdx.x; i < size; i += THREADS) list[i] = 0;
  __syncthreads();
  for (int k = 2; k <= size; k *= 2)
    for (int j = k / 2; j > 0; j /= 2) {
      for (int i = threadIdx.x; i < size / 2; i += THREADS) {
        const int a = 2 * i - (i & (j - 1)), b = a + j;
        const uint64_t x = list[a], y = list[b];
        if ((x < y) == ((a & k) == 0)) list[a] = y, list[b] = x;
      }
      __syncthreads();
    }
}

template <typename E> struct Row {
  const E* x;
  int V;
  double top, inv_t;
  int fixed;
  __device__ __forceinline__ uint32_t key(int i) const { return key_of(to_f32<E>(x[i])); }
  __device__ __forceinline__ double weight(uint32_t k) const { return exp(((double)number_of(k) - top) * inv_t); }
  __device__ __forceinline__ uint64_t whole(double w) const { return (uint64_t)(w * (double)(1ull << fixed) + 0.5); }
};

// How far a search has come: the cut lies among the places from `from` on whose keys are within lo .. hi, and
// `above` (tokens or weight) lies over them.
struct Search {
  bool by_weight;
  double target;      // tokens or (whole) weight to reach
  uint64_t from;      // the cut so far
};

// The bin that holds the cut: the first whose running sum reaches the target; above: the sum before it.
__device__ __forceinline__ int find_bin(Shared& S, const Search& q, uint64_t& above, uint32_t& in_bin) {
  const int t = threadIdx.x;
  const uint64_t v = q.by_weight ? S.mass[t] : S.count[t];
  uint64_t all;
  const uint64_t upto = above + group_scan(v, S.wave64, &all);
  if (t == 0) S.found = BINS - 1;
  __syncthreads();
  if ((double)upto >= q.target && S.count[t] > 0) atomicMin(&S.found, t);
  __syncthreads();
  const int bin = S.found;
  if (t == bin) S.hit = upto - v;
  __syncthreads();
  above = S.hit;
  in_bin = S.count[bin];
  __syncthreads();
  return bin;
}

// Narrows q.from down to the cut.  total: the weight of what q.from keeps, known afterwards where it is by_weight
// and share below 1 (target is set from it).
template <typename E>
__device__ void search_cut(Shared& S, const Row<E>& row, Search& q, double share, float lowest) {
  const int t = threadIdx.x;
  const float top = (float)row.top;
  float range = top - lowest;
  if (q.by_weight) range = fminf(range, (float)(45.0 / row.inv_t));   // (less is less than 2^-64 of the largest)
  const float steps = range > 0.0f ? BINS / range : 0.0f;
  const auto bin_of = [&](uint32_t key) { return (int)fminf((top - number_of(key)) * steps, (float)(BINS - 1)); };
  S.mass[t] = 0, S.count[t] = 0;
  __syncthreads();
  // (the last bin holds all that is far below: it is added up in registers)
  uint64_t far_mass = 0;
  uint32_t far_count = 0;
#pragma unroll 4
  for (int i = t; i < row.V; i += THREADS) {
    const uint32_t key = row.key(i);
    if (key <= DEAD || place_of(key, i) < q.from) continue;
    const int bin = bin_of(key);
    const uint64_t m = q.by_weight ? row.whole(row.weight(key)) : 0;
    if (bin == BINS - 1) {
      far_mass += m;
      ++far_count;
    } else {
      if (q.by_weight) atomicAdd(reinterpret_cast<unsigned long long*>(&S.mass[bin]), (unsigned long long)m);
      atomicAdd(&S.count[bin], 1u);
    }
  }
  if (far_count) {
    atomicAdd(reinterpret_cast<unsigned long long*>(&S.mass[BINS - 1]), (unsigned long long)far_mass);
    atomicAdd(&S.count[BINS - 1], far_count);
  }
  __syncthreads();
  uint64_t all;
  group_scan(q.by_weight ? S.mass[t] : (uint64_t)S.count[t], S.wave64, &all);
  if (q.by_weight) q.target = share * (double)all;
  else if (q.target >= (double)all) return;   // (everything stays)
  uint64_t above = 0;
  uint32_t in_bin;
  const int bin = find_bin(S, q, above, in_bin);

  // which keys are in it
  uint32_t lo = 0, hi = 0xffffffffu;
  bool first_level = true;
  while (in_bin > CAP) {
    if (first_level) {
      uint32_t most = 0, least = 0xffffffffu;
      for (int i = t; i < row.V; i += THREADS) {
        const uint32_t key = row.key(i);
        if (key <= DEAD || place_of(key, i) < q.from || bin_of(key) != bin) continue;
        most = max(most, key), least = min(least, key);
      }
      hi = (uint32_t)group_max(most, S.wave64);
      lo = ~(uint32_t)group_max((uint32_t)~least, S.wave64);
      first_level = false;
    }
    if (lo == hi) break;
    int shift = 0;
    while ((hi - lo) >> shift >= BINS) ++shift;
    __syncthreads();
    S.mass[t] = 0, S.count[t] = 0;
    __syncthreads();
    for (int i = t; i < row.V; i += THREADS) {
      const uint32_t key = row.key(i);
      if (key < lo || key > hi || key <= DEAD || place_of(key, i) < q.from) continue;
      const int b = (hi - key) >> shift;
      if (q.by_weight) atomicAdd(reinterpret_cast<unsigned long long*>(&S.mass[b]), (unsigned long long)row.whole(row.weight(key)));
      atomicAdd(&S.count[b], 1u);
    }
    __syncthreads();
    const int b = find_bin(S, q, above, in_bin);
    const uint32_t new_hi = hi - ((uint32_t)b << shift);
    const uint32_t width = (1u << shift) - 1;
    lo = new_hi - lo > width ? new_hi - width : lo;
    hi = new_hi;
  }

  if (in_bin > CAP) {
    // one number, many times: the cut is the r-th of them in order of their index
    const uint64_t m = q.by_weight ? row.whole(row.weight(hi)) : 1;
    const double r_exact = m ? ceil((q.target - (double)above) / (double)m) : (double)in_bin;
    const uint32_t r = (uint32_t)fmin(fmax(r_exact, 1.0), (double)in_bin);
    // in pieces of the row, one a wave at a time
    uint32_t before = 0;
    const int wave = t >> 6, lane = t & 63;
    if (t == 0) S.hit = 0;
    for (int i0 = 0; i0 < row.V; i0 += THREADS) {
      const int i = i0 + t;
      bool is = false;
      if (i < row.V) {
        const uint32_t key = row.key(i);
        is = key == hi && place_of(key, i) >= q.from;
      }
      const uint64_t mine = __ballot(is);
      __syncthreads();
      if (lane == 0) S.count[wave] = __popcll(mine);
      __syncthreads();
      uint32_t rank = before + __popcll(mine & ((1ull << lane) - 1)), all_here = 0;
      for (int w = 0; w < WAVES; ++w) {
        rank += w < wave ? S.count[w] : 0;
        all_here += S.count[w];
      }
      if (is && rank == r - 1) S.hit = place_of(hi, i);
      before += all_here;
      if (before >= r) break;   // (the same for all)
    }
    __syncthreads();
    q.from = S.hit;
    __syncthreads();
    return;
  }

  // the bin, sorted
  if (t == 0) S.n = 0;
  __syncthreads();
  for (int i = t; i < row.V; i += THREADS) {
    const uint32_t key = row.key(i);
    if (key <= DEAD || place_of(key, i) < q.from) continue;
    if (first_level ? bin_of(key) != bin : key < lo || key > hi) continue;
    const uint32_t at = atomicAdd(&S.n, 1u);
    if (at < CAP) S.list[at] = place_of(key, i);
  }
  __syncthreads();
  const int n = min((int)S.n, CAP);
  sort_list(S.list, n);
  if (t == 0) S.hit = 0;
  uint64_t before = above;
  for (int i0 = 0; i0 < n; i0 += THREADS) {
    const int i = i0 + t;
    const uint64_t m = i >= n ? 0 : q.by_weight ? row.whole(row.weight((uint32_t)(S.list[i] >> 32))) : 1;
    uint64_t here;
    const uint64_t upto = before + group_scan(m, S.wave64, &here);
    // stays if what is before it does not reach the target; the very first stays anyway
    const bool stays = i < n && ((double)(upto - m) < q.target || (i == 0 && above == 0));
    const uint64_t last = group_max(stays ? ~S.list[i] : 0, S.wave64);   // the lowest place that stays
    if (last) q.from = ~last;
    before += here;
  }
  __syncthreads();
}

template <typename E> __global__ __launch_bounds__(THREADS) void oscar_sample_kernel(SampleParams P) {
  __shared__ Shared S;
  const int b = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6, V = P.V;
  Row<E> row;
  row.x = reinterpret_cast<const E*>(P.logits) + (int64_t)b * P.stride;
  row.V = V;
  row.fixed = P.fixed;
  float* probs = P.probs ? P.probs + (int64_t)b * V : nullptr;

  // the largest logit, every thread's largest, and the lowest above -inf
  uint64_t best = 0;
  uint32_t least = 0xffffffffu;
#pragma unroll 8
  for (int i = t; i < V; i += THREADS) {
    const uint32_t key = row.key(i);
    const uint64_t at = place_of(key, i);
    best = at > best ? at : best;
    least = key > DEAD ? min(least, key) : least;
  }
  const uint32_t mine = (uint32_t)(best >> 32);
  best = group_max(best, S.wave64);
  const uint32_t top_key = (uint32_t)(best >> 32);
  const bool any = top_key > DEAD;
  const float temp = P.temperature ? P.temperature[b] : 1.0f;
  const float p = P.top_p ? P.top_p[b] : 1.0f, m = P.min_p ? P.min_p[b] : 0.0f;
  const int k = P.top_k ? P.top_k[b] : 0;
  const float u = P.u[b];
  if (!any || !(temp > 0.0f) || k == 1 || m > 1.0f || p <= 0.0f) {   // one token, or none
    const int token = any ? (int)~(uint32_t)best : 0;
    if (probs)
      for (int i = t; i < V; i += THREADS) probs[i] = any && i == token ? 1.0f : 0.0f;
    if (t == 0) P.tokens[b] = token;
    return;
  }
  row.top = (double)number_of(top_key);
  row.inv_t = 1.0 / (double)temp;
  const double from0 = u > 0.0f ? (double)u : 0.0;

  bool few = k > 0 && k <= THREADS;   // (of what can stay)
  if (few) {
    uint32_t bound = 0;   // the k-th largest of the threads' largest
#pragma unroll 1
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t next = bound | 1u << bit;
      if (__syncthreads_count(mine >= next) >= k) bound = next;
    }
    bound = max(bound, DEAD + 1);
    if (t == 0) S.n = 0;
    __syncthreads();
#pragma unroll 8
    for (int i = t; i < V; i += THREADS) {
      const uint32_t key = row.key(i);
      if (key >= bound) {
        const uint32_t at = atomicAdd(&S.n, 1u);
        if (at < CAP) S.list[at] = place_of(key, i);
      }
    }
    if (probs)
      for (int i = t; i < V; i += THREADS) probs[i] = 0.0f;
    __syncthreads();
    few = S.n <= CAP;
  }
  if (few) {
    int n = (int)S.n;
    sort_list(S.list, n);
    n = min(n, k);   // (up to 1024: a token a thread)
    const uint64_t at = t < n ? S.list[t] : 0;
    const double w = t < n ? row.weight((uint32_t)(at >> 32)) : 0.0;
    double sum;
    const double before = group_scan(w, S.wave_f, &sum) - w;
    const bool stays = t < n && (t == 0 || ((!(p < 1.0f) || before < (double)p * sum) && !(w < (double)m)));
    n = __syncthreads_count(stays);
    // in order of the index
    if (t < n) S.list[t] = ~((uint64_t)(uint32_t)~(uint32_t)at << 32 | (uint32_t)(at >> 32));
    __syncthreads();
    sort_list(S.list, n);
    const uint64_t x = t < n ? ~S.list[t] : 0;
    const double y = t < n ? row.weight((uint32_t)x) : 0.0;
    const double upto = group_scan(y, S.wave_f, &sum);
    if (t == 0) S.found = n - 1;
    __syncthreads();
    if (t < n && upto > from0 * sum) atomicMin(&S.found, t);
    __syncthreads();
    if (t == S.found) P.tokens[b] = (int)(x >> 32);
    if (probs && t < n) probs[x >> 32] = (float)(y / sum);
    return;
  }

  Search q = {false, 0.0, (uint64_t)(DEAD + 1) << 32};
  const float lowest = number_of(~(uint32_t)group_max((uint32_t)~least, S.wave64));
  if (k > 0 && k < V) {
    q.target = (double)k;
    search_cut<E>(S, row, q, 0.0, lowest);
  }
  if (p < 1.0f) {
    q.by_weight = true;
    search_cut<E>(S, row, q, (double)p, lowest);
  }

  // weights of what stays, in pieces of whole waves
  const int piece = 64 * ((V + 64 * BINS - 1) / (64 * BINS)), pieces = (V + piece - 1) / piece;
  const auto weight_at = [&](int i) {
    if (i >= V) return 0.0;
    const uint32_t key = row.key(i);
    if (key <= DEAD || place_of(key, i) < q.from) return 0.0;
    const double w = row.weight(key);
    return w < (double)m ? 0.0 : w;
  };
  __syncthreads();
  for (int c = wave; c < pieces; c += WAVES) {
    double w = 0.0;
    for (int j = 0; j < piece; j += 64) w += weight_at(c * piece + j + lane);
    w = wave_scan(w);
    if (lane == 63) S.part[c] = w;
  }
  __syncthreads();
  double sum;
  const double upto = group_scan(t < pieces ? S.part[t] : 0.0, S.wave_f, &sum);
  const double target = from0 * sum;
  if (t == 0) S.found = pieces, S.n = 0;
  __syncthreads();
  if (t < pieces && S.part[t] > 0.0) {
    if (upto > target) atomicMin(&S.found, t);
    atomicMax(&S.n, (uint32_t)t);
  }
  __syncthreads();
  const bool passed = S.found < pieces;
  const int c = passed ? S.found : (int)S.n;   // (if rounding lets none pass: the last with any weight)
  if (t == c) S.hit = __builtin_bit_cast(uint64_t, upto - S.part[c]);
  __syncthreads();
  if (wave == 0) {
    double before = __builtin_bit_cast(double, S.hit);
    int token = -1, last = 0;
    for (int j = 0; j < piece && token < 0; j += 64) {
      const int i = c * piece + j + lane;
      const double w = weight_at(i);
      const double here = wave_scan(w);
      const uint64_t past = __ballot(w > 0.0 && before + here > target), some = __ballot(w > 0.0);
      if (some) last = c * piece + j + 63 - __builtin_clzll(some);
      if (past) token = c * piece + j + __builtin_ctzll(past);
      before += __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(__builtin_bit_cast(uint64_t, here) >> 32), 63) << 32 |
                                               (uint32_t)__builtin_amdgcn_readlane((int)__builtin_bit_cast(uint64_t, here), 63));
    }
    if (lane == 0) P.tokens[b] = token < 0 ? last : token;
  }
  if (probs)
    for (int i = t; i < V; i += THREADS) probs[i] = (float)(weight_at(i) / sum);
}

}  // namespace

extern "C" int oscar_sample(const void* logits, int64_t row_stride, int32_t batch, int32_t vocab, int32_t dtype,
                            const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                            const float* u, int32_t* tokens, float* probs, void* stream) {
  if (dtype != OSCAR_F32 && dtype != OSCAR_BF16 && dtype != OSCAR_F16) return OSCAR_ERR_INVALID_ARG;
  if (batch < 0 || vocab < 1 || vocab > OSCAR_VERIFY_MAX_VOCAB || (batch > 1 && row_stride < vocab)) return OSCAR_ERR_INVALID_ARG;
  if ((int64_t)batch * THREADS > UINT32_MAX) return OSCAR_ERR_INVALID_ARG;   // (a grid's threads are counted in 32 bits)
  if (batch == 0) return OSCAR_OK;
  if (!logits || !u || !tokens) return OSCAR_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == OSCAR_F32 ? 4 : 2) != 0) return OSCAR_ERR_INVALID_ARG;
  SampleParams P = {logits, row_stride, vocab, 0, temperature, top_p, min_p, u, top_k, tokens, probs};
  P.fixed = 62;
  while ((int64_t)1 << (62 - P.fixed) < vocab) --P.fixed;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (dtype == OSCAR_F32)
    hipLaunchKernelGGL((oscar_sample_kernel<float>), dim3(batch), dim3(THREADS), 0, st, P);
  else if (dtype == OSCAR_BF16)
    hipLaunchKernelGGL((oscar_sample_kernel<__hip_bfloat16>), dim3(batch), dim3(THREADS), 0, st, P);
  else
    hipLaunchKernelGGL((oscar_sample_kernel<__half>), dim3(batch), dim3(THREADS), 0, st, P);
  if (hipGetLastError() != hipSuccess) return OSCAR_ERR_HIP;
  return OSCAR_OK;
}
