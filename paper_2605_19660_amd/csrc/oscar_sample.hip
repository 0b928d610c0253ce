// oscar_sample: a token from every row of logits, from given random numbers.
//
//   w_i = exp((l_i - max l) / temperature); in order of falling (l_i, -i):
//   the first top_k; of those the first whose weights reach top_p of their sum; of those the ones with w >= min_p
//   token = the smallest i with w_0 + .. + w_i > u * sum over what stays
//
// Every filter keeps a prefix of that order, so that what stays is everything from one pair (logit, index) on: the pair
// is held as one 64-bit number, (logit as an ordered integer, ~index), and the search is for that number, the cut.
// Weights are 64-bit floats, to 2^-40 of themselves and better: the exponential is good to 2^-45 (by a table; a series
// good to 2^-51 takes 80 us where it takes 72, 64 draws of 128003), its argument to half a step, which counts far below the largest.
// Where many are added by atomics they count as whole multiples of a power of two, so that no order of additions changes a bit:
// 2^-49 of a chunk's largest (8192 of them at most: 2^-37 of it), 2^-50 of the row's on its list (4096: 2^-39), 2^-80 of it where one workgroup has the
// row.  Sums are within 2^-36 of the row's; settings and random numbers have 24 bits.
//
// A row is taken in chunks, so that few rows still fill the chip, and logits lie in bins of equal steps (at most
// temperature * 45 / 1024), counted from 0 so that chunks' bins lie on one grid:
//   1. every chunk: its largest logit, and the running sums (of tokens for top_k, else of weights, in 64 bits) over
//      the 1024 bins below it;
//   2. the row's running sums are added up, each chunk's shifted by whole bins and scaled by one factor, and the bins found
//      in which the cuts lie: with few chunks by each of them, else by a workgroup a row in a launch of its own;
//   3. every chunk puts its logits in those bins (with top_k: in those and above) on the row's list;
//   4. a workgroup a row: sorts the list, finds the cut in it, what stays of every chunk (running sums above the list,
//      the list's members one by one), the chunk the token is in, and in it the token;
//   5. with probs, every chunk: its probabilities.
// A row whose list does not fit (thousands of equal logits at the cut) or with a top_k past 1024 is searched by
// one workgroup, which splits bins until they fit or hold one number.
//
// What bounds it: one row of 32000 with top_p takes 24 us, a chain of dependent steps in three launches (6.6, 7.1 and 9.6):
// loads that wait for the launch before, scans over a workgroup, a sort.  64 rows of 128003 with mixed settings and
// probabilities take 71 us, 21.1 bins, 7.8 to find, 9.6 list, 15.7 draw, 16.8 probabilities: the rows are read three times
// (8 us where nothing else is done, 5 TB/s; past the first time out of the caches), the bins are bound by vector instructions
// (40 a logit, half of them its exponential), the draw by its longest list.
#include "oscar_common.h"

namespace {

constexpr int THREADS = 1024, WAVES = 16;
constexpr int BINS = 1024;
constexpr int CAP = 4096;                  // numbers sorted in LDS
constexpr uint32_t DEAD = 0x007fffffu;     // key of -inf
constexpr int CHUNK_BITS = 49;             // binary places of a weight in a chunk's sums (2^13 of them at most)
constexpr int LIST_BITS = 50;              // of a member of the list (2^12)

// What the launches leave of a row.
struct RowState {
  uint32_t n;         // members of the list
  int lo, hi;         // bins on the list
  int kind;           // of what stays: see the launch that draws
  int first;          // cell of the row's largest logit
  double above, total;   // weights above the list, and of all
  uint64_t cut;
  double sum;         // weights of what stays
};
enum { ONE_TOKEN, NO_TOKEN, BY_CUT, DONE };

struct SampleParams {
  const void* logits;
  int64_t stride;
  int V;               // vocabulary
  int chunks, chunk;   // of a row, and their size
  const float *temperature, *top_p, *min_p, *u;
  const int32_t* top_k;
  int32_t* tokens;
  float* probs;
  uint64_t* best;      // [batch][chunks]: place of the largest logit
  uint64_t* cum;       // [batch][chunks][BINS]: running sums
  RowState* rows;      // [batch]
  uint64_t* list;      // [batch][CAP]
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

// 2^z 2^PLACES, z <= 0 or a little above, to 2^-51 of itself: 2^n 2^f with |f| <= 1/2, the series of 2^f up to f^13
// ((ln 2)^k / k!; the next term is below 2^-57).
template <int PLACES = 0> __device__ __forceinline__ double power_of_2(double z) {
  z = fmax(z, -1200.0);
  const double n = __builtin_rint(z), f = z - n;
  double s = 0x1.816193166d0f9p-40;
  s = fma(s, f, 0x1.c3bd650fc2986p-36);
  s = fma(s, f, 0x1.e8cac7351bb25p-32);
  s = fma(s, f, 0x1.e4cf5158b8ecap-28);
  s = fma(s, f, 0x1.b5253d395e7c4p-24);
  s = fma(s, f, 0x1.62c0223a5c824p-20);
  s = fma(s, f, 0x1.ffcbfc588b0c7p-17);
  s = fma(s, f, 0x1.430912f86c787p-13);
  s = fma(s, f, 0x1.5d87fe78a6731p-10);
  s = fma(s, f, 0x1.3b2ab6fba4e77p-7);
  s = fma(s, f, 0x1.c6b08d704a0c0p-5);
  s = fma(s, f, 0x1.ebfbdff82c58fp-3);
  s = fma(s, f, 0x1.62e42fefa39efp-1);
  s = fma(s, f, 0x1.0000000000000p+0);
  return __builtin_amdgcn_ldexp(s, (int)n + PLACES);
}
// The same, to 2^-45, by a table of 2^(i / 32), i < 32: |f| <= 1/64 of a power is left, the series ends with f^5.
__device__ __forceinline__ void fill_powers(double* table) {
  if (threadIdx.x < 32) table[threadIdx.x] = power_of_2((double)threadIdx.x * 0.03125);
}
template <int PLACES> __device__ __forceinline__ double power_of_2(double z, const double* table) {
  z = fmax(z * 32.0, -38400.0);
  const double n = __builtin_rint(z), f = z - n;
  const int i = (int)n;
  const double t = table[i & 31];
  double s = 0x1.5d87fe78a6731p-35;
  s = fma(s, f, 0x1.3b2ab6fba4e77p-27);
  s = fma(s, f, 0x1.c6b08d704a0c0p-20);
  s = fma(s, f, 0x1.ebfbdff82c58fp-13);
  s = fma(s, f, 0x1.62e42fefa39efp-6);
  return __builtin_amdgcn_ldexp(fma(s * f, t, t), (i >> 5) + PLACES);
}
// A number below 2^52, rounded to a whole one.
__device__ __forceinline__ uint64_t whole_of(double x) {
  return __builtin_bit_cast(uint64_t, x + 0x1p52) & ((1ull << 52) - 1);
}

// The lanes' numbers moved up within a wave, 0 where none comes from; four steps inside rows of 16 lanes and two that carry
// a row's last lane on (as permutations through LDS a scan waits for them six times).
template <int CTRL, int ROWS> __device__ __forceinline__ uint64_t moved(uint64_t bits) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(bits >> 32), CTRL, ROWS, 0xf, false);
  return (uint64_t)hi << 32 | lo;
}
template <int CTRL, int ROWS, typename T, typename F> __device__ __forceinline__ T step(T v, F f) {
  return f(v, __builtin_bit_cast(T, moved<CTRL, ROWS>(__builtin_bit_cast(uint64_t, v))));
}
template <typename T, typename F> __device__ __forceinline__ T wave_prefix(T v, F f) {   // f(x, 0) = x
  v = step<0x111, 0xf>(v, f);   // row_shr:1, 2, 4, 8
  v = step<0x112, 0xf>(v, f);
  v = step<0x114, 0xf>(v, f);
  v = step<0x118, 0xf>(v, f);
  v = step<0x142, 0xa>(v, f);   // row_bcast:15 into rows 1 and 3
  return step<0x143, 0xc>(v, f);   // row_bcast:31 into rows 2 and 3
}
template <typename T> __device__ __forceinline__ T wave_scan(T v) {
  return wave_prefix(v, [](T a, T b) { return a + b; });
}
__device__ __forceinline__ double of_last_lane(double v) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)bits, 63), hi = __builtin_amdgcn_readlane((int)(bits >> 32), 63);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Sum over the threads up to this one; all: over all; s[w] is then the wave's sum.  s: WAVES numbers.
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
__device__ __forceinline__ uint64_t group_max(uint64_t v, uint64_t* s) {
  v = wave_prefix(v, [](uint64_t a, uint64_t b) { return b > a ? b : a; });
  __syncthreads();
  if ((threadIdx.x & 63) == 63) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) v = s[w] > v ? s[w] : v;
  return v;
}
// The largest of each half.
__device__ __forceinline__ uint64_t group_max_halves(uint32_t upper, uint32_t lower, uint64_t* s) {
  const auto most = [](uint64_t a, uint64_t b) { return (uint64_t)max((uint32_t)(a >> 32), (uint32_t)(b >> 32)) << 32 | max((uint32_t)a, (uint32_t)b); };
  uint64_t v = wave_prefix((uint64_t)upper << 32 | lower, most);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) v = most(v, s[w]);
  return v;
}

// One addition in LDS a wave, one minimum a wave (of 1024 threads at one address each waits for all before it: 3 us).
__device__ __forceinline__ void add_from_wave(uint64_t* to, uint64_t v) {
  v = wave_scan(v);
  if ((threadIdx.x & 63) == 63 && v) atomicAdd(reinterpret_cast<unsigned long long*>(to), (unsigned long long)v);
}
// The lowest thread for which `is`.
__device__ __forceinline__ void first_thread(int* to, bool is) {
  const uint64_t those = __ballot(is);
  if ((threadIdx.x & 63) == 0 && those) atomicMin(to, (int)threadIdx.x + __builtin_ctzll(those));
}
__device__ __forceinline__ void last_thread(uint32_t* to, bool is) {
  const uint64_t those = __ballot(is);
  if ((threadIdx.x & 63) == 0 && those) atomicMax(to, threadIdx.x + 63 - __builtin_clzll(those));
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

// Falling order of S.list[0 .. n), all different, by the workgroup; returns with the list in place for all.  Up to 256 numbers
// each counts those above it; more are dealt into bins of equal steps (LOGITS: of the logits they are places of), where each
// counts its own bin.  Where one bin gets many they are sorted by exchanges, a barrier a step.  (Two sorts a draw with top_k of
// one row of 128003: top_k 1000, exchanged 56 us, by bins 39; 400, counted 40, by bins 36; 200 31 and 34; 50 25 and 33.)
template <bool LOGITS> __device__ __forceinline__ void sort_list(Shared& S, int n) {
  uint64_t* list = S.list;
  if (n <= THREADS / 4) {
    const uint64_t mine = threadIdx.x < n ? list[threadIdx.x] : 0;
    int above = 0;
    if (threadIdx.x < n) {
#pragma unroll 8
      for (int i = 0; i < n; ++i) above += list[i] > mine ? 1 : 0;
    }
    __syncthreads();
    if (threadIdx.x < n) list[above] = mine;
    __syncthreads();
    return;
  }
  {
    const int t = threadIdx.x;
    uint64_t x[CAP / THREADS], most = 0, least = ~0ull;
#pragma unroll
    for (int i = 0; i < CAP / THREADS; ++i) {
      x[i] = i * THREADS + t < n ? list[i * THREADS + t] : 0;
      if (i * THREADS + t < n) most = x[i] > most ? x[i] : most, least = x[i] < least ? x[i] : least;
    }
    S.count[t] = 0;
    most = group_max(most, S.wave64);
    least = ~group_max(~least, S.wave64);
    const int shift = max(54 - __builtin_clzll((most - least) | 1), 0);   // (1024 bins)
    const float top = number_of((uint32_t)(most >> 32)), range = top - number_of((uint32_t)(least >> 32));
    const bool logits = LOGITS && range > 0.0f && range < INFINITY;
    const auto bin_of = [&](uint64_t place) {
      return logits ? (int)((top - number_of((uint32_t)(place >> 32))) / range * (BINS - 1)) : (int)((most - place) >> shift);
    };
    uint32_t at[CAP / THREADS];
#pragma unroll
    for (int i = 0; i < CAP / THREADS; ++i) at[i] = i * THREADS + t < n ? atomicAdd(&S.count[bin_of(x[i])], 1u) : 0;
    __syncthreads();
    const uint32_t here = S.count[t];
    uint64_t all;
    const uint32_t upto = (uint32_t)group_scan((uint64_t)here, S.wave64, &all);
    S.count[t] = upto;
    if (!__syncthreads_or(here > 32)) {
      int from[CAP / THREADS], to[CAP / THREADS];
#pragma unroll
      for (int i = 0; i < CAP / THREADS; ++i) {
        if (i * THREADS + t >= n) continue;
        const int bin = bin_of(x[i]);
        from[i] = bin ? S.count[bin - 1] : 0, to[i] = S.count[bin];
        list[from[i] + at[i]] = x[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < CAP / THREADS; ++i) {
        if (i * THREADS + t >= n) continue;
        at[i] = from[i];
        for (int j = from[i]; j < to[i]; ++j) at[i] += list[j] > x[i] ? 1 : 0;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < CAP / THREADS; ++i)
        if (i * THREADS + t < n) list[at[i]] = x[i];
      __syncthreads();
      return;
    }
  }
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
  double top, scale;   // scale: log2(e) / temperature
  const double* powers;
  __device__ __forceinline__ uint32_t key(int i) const { return key_of(to_f32<E>(x[i])); }
  __device__ __forceinline__ double weight(uint32_t k) const { return power_of_2<0>(((double)number_of(k) - top) * scale, powers); }
};

// Weights of a whole row are added up in two whole numbers, of multiples of 2^-40 and of what is left in multiples of 2^-80
// (2^22 of either stay below 2^63): millions of tokens of 2^-42 beside one of 1 are not lost.
__device__ __forceinline__ void split_weight(double w, uint64_t& high, uint64_t& low) {
  const double x = w * 0x1p40, whole = floor(x);
  high = whole_of(whole), low = whole_of((x - whole) * 0x1p40);
}
__device__ __forceinline__ double joined_weight(uint64_t high, uint64_t low) { return (double)high * 0x1p-40 + (double)low * 0x1p-80; }

// How far a search has come: the cut lies among the places from `from` on whose keys are within lo .. hi, and
// `above` (tokens or weight) lies over them.
struct Search {
  bool by_weight;
  double target;      // tokens or weight to reach
  uint64_t from;      // the cut so far
};

// What a search has in bin t: tokens, or their weight.  The weights' lower parts lie where the list is not yet.
__device__ __forceinline__ double in_bin_of(const Shared& S, const Search& q, int t) {
  return q.by_weight ? joined_weight(S.mass[t], S.list[t]) : (double)S.count[t];
}
__device__ __forceinline__ void clear_bins(Shared& S) {
  S.mass[threadIdx.x] = 0, S.list[threadIdx.x] = 0, S.count[threadIdx.x] = 0;
}
__device__ __forceinline__ void add_to_bin(Shared& S, int bin, double w) {
  uint64_t high, low;
  split_weight(w, high, low);
  atomicAdd(reinterpret_cast<unsigned long long*>(&S.mass[bin]), (unsigned long long)high);
  atomicAdd(reinterpret_cast<unsigned long long*>(&S.list[bin]), (unsigned long long)low);
}

// The bin that holds the cut: the first whose running sum reaches the target; above: the sum before it.
__device__ __forceinline__ int find_bin(Shared& S, const Search& q, double& above, uint32_t& in_bin) {
  const int t = threadIdx.x;
  const double v = in_bin_of(S, q, t);
  double all;
  const double upto = above + group_scan(v, S.wave_f, &all);
  if (t == 0) S.found = BINS - 1;
  __syncthreads();
  first_thread(&S.found, upto >= q.target && S.count[t] > 0);
  __syncthreads();
  const int bin = S.found;
  if (t == bin) S.hit = __builtin_bit_cast(uint64_t, upto - v);
  __syncthreads();
  above = __builtin_bit_cast(double, S.hit);
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
  if (q.by_weight) range = fminf(range, (float)(65.0 / row.scale));   // (less is less than 2^-64 of the largest)
  const float steps = range > 0.0f ? BINS / range : 0.0f;
  const auto bin_of = [&](uint32_t key) { return (int)fminf((top - number_of(key)) * steps, (float)(BINS - 1)); };
  clear_bins(S);
  __syncthreads();
  // (the last bin holds all that is far below: it is added up in registers)
  uint64_t far_high = 0, far_low = 0;
  uint32_t far_count = 0;
#pragma unroll 4
  for (int i = t; i < row.V; i += THREADS) {
    const uint32_t key = row.key(i);
    if (key <= DEAD || place_of(key, i) < q.from) continue;
    const int bin = bin_of(key);
    if (bin == BINS - 1) {
      if (q.by_weight) {
        uint64_t high, low;
        split_weight(row.weight(key), high, low);
        far_high += high, far_low += low;
      }
      ++far_count;
    } else {
      if (q.by_weight) add_to_bin(S, bin, row.weight(key));
      atomicAdd(&S.count[bin], 1u);
    }
  }
  add_from_wave(&S.mass[BINS - 1], far_high);
  add_from_wave(&S.list[BINS - 1], far_low);
  far_count = (uint32_t)wave_scan((uint64_t)far_count);
  if ((t & 63) == 63 && far_count) atomicAdd(&S.count[BINS - 1], far_count);
  __syncthreads();
  double all;
  group_scan(in_bin_of(S, q, t), S.wave_f, &all);
  if (q.by_weight) q.target = share * all;
  else if (q.target >= all) return;   // (everything stays)
  double above = 0.0;
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
    clear_bins(S);
    __syncthreads();
    for (int i = t; i < row.V; i += THREADS) {
      const uint32_t key = row.key(i);
      if (key < lo || key > hi || key <= DEAD || place_of(key, i) < q.from) continue;
      const int b = (hi - key) >> shift;
      if (q.by_weight) add_to_bin(S, b, row.weight(key));
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
    const double m = q.by_weight ? row.weight(hi) : 1.0;
    const double r_exact = m > 0.0 ? ceil((q.target - above) / m) : (double)in_bin;
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
  sort_list<true>(S, n);
  if (t == 0) S.hit = 0;
  double before = above;
  for (int i0 = 0; i0 < n; i0 += THREADS) {
    const int i = i0 + t;
    const double m = i >= n ? 0.0 : q.by_weight ? row.weight((uint32_t)(S.list[i] >> 32)) : 1.0;
    double here;
    const double upto = before + group_scan(m, S.wave_f, &here);
    // stays if what is before it does not reach the target; the very first stays anyway
    const bool stays = i < n && (upto - m < q.target || (i == 0 && above == 0.0));
    const uint64_t last = group_max(stays ? ~S.list[i] : 0, S.wave64);   // the lowest place that stays
    if (last) q.from = ~last;
    before += here;
  }
  __syncthreads();
}

// A row by one workgroup, whatever its list would be.
template <typename E> __device__ void whole_row(Shared& S, const SampleParams& P, const Row<E>& row, int b, int k, float p, float m, double from0) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, V = P.V;
  float* probs = P.probs ? P.probs + (int64_t)b * V : nullptr;
  uint32_t least = 0xffffffffu;
#pragma unroll 8
  for (int i = t; i < V; i += THREADS) {
    const uint32_t key = row.key(i);
    least = key > DEAD ? min(least, key) : least;
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
  first_thread(&S.found, t < pieces && S.part[t] > 0.0 && upto > target);
  last_thread(&S.n, t < pieces && S.part[t] > 0.0);
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
      before += of_last_lane(here);
    }
    if (lane == 0) P.tokens[b] = token < 0 ? last : token;
  }
  if (probs)
    for (int i = t; i < V; i += THREADS) probs[i] = (float)(weight_at(i) / sum);
}

// How a row is drawn.
struct Settings {
  float temp, p, m;
  int k;
  double u;
  bool one;       // the largest logit
  bool by_count;  // top_k that fits the list: bins count tokens
  bool whole;     // top_k that does not: one workgroup
  bool cuts;      // else: whether top_p or min_p cut
  float width, grid;   // of a bin, and bins a unit
};
__device__ __forceinline__ Settings settings(const SampleParams& P, int b) {
  Settings s;
  s.temp = P.temperature ? P.temperature[b] : 1.0f;
  s.p = P.top_p ? P.top_p[b] : 1.0f;
  s.m = P.min_p ? P.min_p[b] : 0.0f;
  s.k = P.top_k ? P.top_k[b] : 0;
  const float u = P.u[b];
  s.u = u > 0.0f ? (double)u : 0.0;
  s.one = !(s.temp > 0.0f) || s.k == 1 || s.m > 1.0f || s.p <= 0.0f;
  s.by_count = s.k > 0 && s.k <= THREADS;
  s.whole = !s.by_count && s.k > 0 && s.k < P.V;
  s.cuts = s.p < 1.0f || s.m > 0.0f;
  // weights fall to 2^-64 over the bins, or logits by 64, whichever is less: a high temperature spreads weights over
  // few of the former
  s.width = fminf(fmaxf(45.0f * s.temp, 1e-25f), 64.0f) * (1.0f / BINS);
  s.grid = 1.0f / s.width;
  return s;
}
// The grid's cell of a logit; cells fall with it.
__device__ __forceinline__ int cell_of(float x, float grid) { return -(int)floorf(__builtin_amdgcn_fmed3f(x * grid, -0x1p30f, 0x1p30f)); }
// Cells are narrower than a float's steps from 2^24 on.  A row whose largest logit is past ROW_GRID is searched by one
// workgroup; a chunk whose largest is past CHUNK_GRID has everything in its last bin (far below such a row's bins).
constexpr float ROW_GRID = 0x1p21f, CHUNK_GRID = 0x1p22f;
__device__ __forceinline__ bool on_grid(float top, float grid, float end) { return fabsf(top * grid) < end; }
// The bin of a logit under a cell of the grid (its negative, as a float): whole numbers below 2^24, or far above BINS.
__device__ __forceinline__ int bin_under(float first, float x, float grid) {
  return (int)fminf(first - floorf(x * grid), (float)(BINS - 1));
}
// A chunk's logits, a thread's 1024 apart, as numbers that have an order: NaN as -inf, +inf as the largest; -inf behind
// the row's end.
template <typename E, int PER> __device__ __forceinline__ void load_row(const SampleParams& P, int b, int c, float* x) {
  const E* from = reinterpret_cast<const E*>(P.logits) + (int64_t)b * P.stride;
  const int i0 = c * (PER * THREADS) + threadIdx.x;
  // (all on the way before the first is looked at: no branch around a load, 1.5 .. 3 us a launch.  As vectors of 16 bytes,
  // at rows of odd lengths, the launches take 1 .. 2 us longer)
  E raw[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) raw[e] = from[min(i0 + e * THREADS, P.V - 1)];
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const float v = to_f32<E>(raw[e]);
    x[e] = i0 + e * THREADS < P.V && v == v ? fminf(v, 3.402823466e38f) : -INFINITY;
  }
}

template <typename E, int PER> __global__ __launch_bounds__(THREADS, 8) void oscar_sample_bins_kernel(SampleParams P) {
  __shared__ uint64_t s_bin[BINS], s_wave[WAVES];
  __shared__ double s_power[32];
  const int b = blockIdx.y, c = blockIdx.x, t = threadIdx.x;
  float x[PER];
  load_row<E, PER>(P, b, c, x);
  float most = x[0];
#pragma unroll
  for (int e = 1; e < PER; ++e) most = fmaxf(most, x[e]);
  const Settings s = settings(P, b);
  s_bin[t] = 0;
  fill_powers(s_power);
  uint32_t first_most = 0;   // of the largest
#pragma unroll
  for (int e = PER - 1; e >= 0; --e) first_most = x[e] == most ? c * (PER * THREADS) + e * THREADS + t : first_most;
  const uint64_t best = group_max(place_of(key_of(most), first_most), s_wave);
  const int64_t chunk = (int64_t)b * P.chunks + c;
  if (t == 0) {
    P.best[chunk] = best;
    if (c == 0) P.rows[b].n = 0;
  }
  const float top = number_of((uint32_t)(best >> 32));
  if (s.one || s.whole || (uint32_t)(best >> 32) <= DEAD) return;
  const float first = on_grid(top, s.grid, CHUNK_GRID) ? floorf(top * s.grid) : INFINITY;
  uint64_t mine = 0;   // the last bin's, and without cuts everything
  if (s.by_count) {
    uint32_t far = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int bin = bin_under(first, x[e], s.grid);
      if (bin < BINS - 1) atomicAdd(reinterpret_cast<uint32_t*>(&s_bin[bin]), 1u);
      far += bin == BINS - 1 && x[e] > -INFINITY ? 1 : 0;
    }
    mine = far;
  } else {
    const double ref = (double)top, scale = 1.4426950408889634 / (double)s.temp;
    uint64_t w[PER];   // (without branches: the exponentials' steps wait for each other, and side by side they do not; -inf: 0)
#pragma unroll
    for (int e = 0; e < PER; ++e) w[e] = whole_of(power_of_2<CHUNK_BITS>(((double)x[e] - ref) * scale, s_power));
    if (s.cuts) {
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const int bin = bin_under(first, x[e], s.grid);
        if (bin < BINS - 1) atomicAdd(reinterpret_cast<unsigned long long*>(&s_bin[bin]), (unsigned long long)w[e]);
        mine += bin == BINS - 1 ? w[e] : 0;
      }
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e) mine += w[e];
    }
  }
  add_from_wave(&s_bin[BINS - 1], mine);
  __syncthreads();
  if (!s.by_count && !s.cuts) {   // (nothing is looked up but their sum)
    if (t == 0) P.cum[chunk * BINS + BINS - 1] = s_bin[BINS - 1];
    return;
  }
  uint64_t all;
  P.cum[chunk * BINS + t] = group_scan(s_bin[t], s_wave, &all);
}

// A row's chunks on one grid: every chunk's first bin in the row's, and what its sums are multiplied by.
struct Chunks {
  int shift[THREADS];      // -1: the chunk has no logit above -inf
  double scale[THREADS];
};
// best: the largest logit (its place) of the chunk with the thread's number.
__device__ __forceinline__ void place_chunk(const Settings& s, uint64_t best, float top, bool is, Chunks& G) {
  const int t = threadIdx.x;
  if (is) {
    const uint32_t key = (uint32_t)(best >> 32);
    const int first = cell_of(number_of(key), s.grid);
    G.shift[t] = key > DEAD ? first - cell_of(top, s.grid) : -1;
    G.scale[t] = s.by_count ? 1.0 : power_of_2<-CHUNK_BITS>(((double)number_of(key) - (double)top) * (1.4426950408889634 / (double)s.temp));
  }
  __syncthreads();
}
// A chunk's running sum up to the row's bin.  (The load does not wait for whether it counts.)
__device__ __forceinline__ double chunk_upto(const SampleParams& P, const Chunks& G, int64_t row_chunk, int c, int bin) {
  const int shift = G.shift[c], own = bin == BINS - 1 ? bin : bin - shift;
  const uint64_t sum = P.cum[(row_chunk + c) * BINS + max(own, 0)];
  return (double)(shift < 0 || own < 0 ? 0 : sum) * (shift < 0 ? 0.0 : G.scale[c]);
}

// The bins that hold the cuts, by a workgroup with a thread a bin.
struct Found {
  int lo, hi;
  double above, total;   // weights above bin lo, and of all
};
struct FindShared {
  Chunks G;
  double cum[BINS];
  int bin;
};
__device__ __forceinline__ Found find_bins(const SampleParams& P, const Settings& s, int b, uint64_t chunk_best, float top, FindShared& F) {
  const int t = threadIdx.x;
  place_chunk(s, chunk_best, top, t < P.chunks, F.G);
  double upto = 0.0;
  for (int q = 0; q < P.chunks; q += 8) {   // (8 on the way at a time)
    double part[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) part[i] = chunk_upto(P, F.G, (int64_t)b * P.chunks, min(q + i, P.chunks - 1), t);
#pragma unroll
    for (int i = 0; i < 8; ++i) upto += q + i < P.chunks ? part[i] : 0.0;
  }
  F.cum[t] = upto;
  if (t == 0) F.bin = BINS - 1;
  __syncthreads();
  Found f = {BINS, -1, 0.0, F.cum[BINS - 1]};
  if (s.by_count || s.p < 1.0f) {
    const double target = s.by_count ? fmin((double)s.k, f.total) : (double)s.p * f.total;
    first_thread(&F.bin, upto >= target);
    __syncthreads();
    f.hi = F.bin;
    f.lo = s.by_count ? 0 : f.hi;
  }
  if (!s.by_count && s.m > 0.0f) {
    // the bins in which weights pass min_p, a little more on either side
    const double x = (double)top + (double)s.temp * log((double)s.m), off = 1e-6 * (fabs((double)top) + fabs(x) + (double)s.temp);
    const int first = cell_of(top, s.grid);
    int from = 0, to = BINS - 1;
    if (fabs(x) < 3e38) {   // (not at a temperature without end)
      from = max(min(cell_of((float)(x + off), s.grid) - first, BINS - 1), 0);
      to = max(min(cell_of((float)(x - off), s.grid) - first, BINS - 1), 0);
    }
    if (to < f.lo)
      f.lo = from, f.hi = to;      // min_p cuts before top_p does
    else if (from <= f.hi)
      f.lo = min(f.lo, from), f.hi = max(f.hi, to);
  }
  f.above = f.lo > 0 ? F.cum[f.lo - 1] : 0.0;
  return f;
}
__device__ __forceinline__ bool has_list(const Settings& s) { return !s.one && !s.whole && (s.by_count || s.cuts); }

__global__ __launch_bounds__(THREADS) void oscar_sample_find_kernel(SampleParams P) {
  __shared__ FindShared F;
  __shared__ uint64_t s_wave[WAVES];
  const int b = blockIdx.x, t = threadIdx.x;
  const uint64_t chunk_best = t < P.chunks ? P.best[(int64_t)b * P.chunks + t] : 0;
  const Settings s = settings(P, b);
  const uint32_t top_key = (uint32_t)(group_max(chunk_best, s_wave) >> 32);
  const float top = number_of(top_key);
  RowState& r = P.rows[b];
  Found f = {0, -1, 0.0, 0.0};   // (no list)
  if (has_list(s) && top_key > DEAD && on_grid(top, s.grid, ROW_GRID)) f = find_bins(P, s, b, chunk_best, top, F);
  if (t == 0) r.lo = f.lo, r.hi = f.hi, r.above = f.above, r.total = f.total, r.first = cell_of(top, s.grid);
}

// FIND: the chunks look for the bins themselves (a launch less; but every chunk reads the sums of all the row's).
template <typename E, int PER, bool FIND> __global__ __launch_bounds__(THREADS, 8) void oscar_sample_list_kernel(SampleParams P) {
  const int b = blockIdx.y, c = blockIdx.x, t = threadIdx.x, lane = t & 63;
  // (what the launch waits for is asked for at once)
  const Settings s = settings(P, b);
  float x[PER];
  int lo, hi, first;
  if constexpr (FIND) {
    __shared__ FindShared F;
    __shared__ uint64_t s_wave[WAVES];
    const uint64_t chunk_best = t < P.chunks ? P.best[(int64_t)b * P.chunks + t] : 0;
    load_row<E, PER>(P, b, c, x);
    if (!has_list(s)) return;
    const uint32_t top_key = (uint32_t)(group_max(chunk_best, s_wave) >> 32);
    const float top = number_of(top_key);
    if (top_key <= DEAD || !on_grid(top, s.grid, ROW_GRID)) return;
    const Found f = find_bins(P, s, b, chunk_best, top, F);
    lo = f.lo, hi = f.hi, first = cell_of(top, s.grid);
    if (c == 0 && t == 0) {
      RowState& r = P.rows[b];
      r.lo = lo, r.hi = hi, r.above = f.above, r.total = f.total;
    }
  } else {
    const RowState& r = P.rows[b];
    lo = r.lo, hi = r.hi, first = r.first;
    if (hi < 0) return;
    load_row<E, PER>(P, b, c, x);
  }
  uint32_t on = 0;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int bin = bin_under(-(float)first, x[e], s.grid);
    on |= (x[e] > -INFINITY && bin >= lo && bin <= hi ? 1u : 0u) << e;
  }
  // a place on the list, a wave at a time
  const uint64_t mine = __popc(on), upto = wave_scan(mine);
  uint32_t at = 0;
  if (lane == 63 && upto) at = atomicAdd(&P.rows[b].n, (uint32_t)upto);
  at = (uint32_t)__builtin_amdgcn_readlane((int)at, 63) + (uint32_t)(upto - mine);
#pragma unroll
  for (int e = 0; e < PER; ++e)
    if (on >> e & 1) {
      if (at < CAP) P.list[(int64_t)b * CAP + at] = place_of(key_of(x[e]), c * (PER * THREADS) + e * THREADS + t);
      ++at;
    }
}

template <typename E, int PER> __global__ __launch_bounds__(THREADS) void oscar_sample_pick_kernel(SampleParams P) {
  __shared__ Shared S;
  __shared__ Chunks G;
  __shared__ double s_power[32];
  const int b = blockIdx.x, t = threadIdx.x, V = P.V;
  const uint64_t chunk_best = t < P.chunks ? P.best[(int64_t)b * P.chunks + t] : 0;
  const Settings s = settings(P, b);
  RowState& R = P.rows[b];
  const RowState r = R;
  uint64_t member[CAP / THREADS];
#pragma unroll
  for (int i = 0; i < CAP / THREADS; ++i) {
    // (what lies behind the list's end is not used; its length is still on its way)
    member[i] = P.list[(int64_t)b * CAP + i * THREADS + t];
  }
  fill_powers(s_power);
  const uint64_t best = group_max(chunk_best, S.wave64);
  const uint32_t top_key = (uint32_t)(best >> 32);
  if (top_key <= DEAD || s.one) {
    if (t == 0) {
      P.tokens[b] = top_key <= DEAD ? 0 : (int)~(uint32_t)best;
      R.kind = top_key <= DEAD ? NO_TOKEN : ONE_TOKEN;
    }
    return;
  }
  const float top = number_of(top_key);
  Row<E> row = {reinterpret_cast<const E*>(P.logits) + (int64_t)b * P.stride, V, (double)top, 1.4426950408889634 / (double)s.temp, s_power};
  const bool listed = s.by_count || s.cuts;
  int n = listed ? (int)min(r.n, (uint32_t)CAP + 1) : 0;
  if (s.whole || !on_grid(top, s.grid, ROW_GRID) || n > CAP) {
    if (t == 0) R.kind = DONE;
    whole_row<E>(S, P, row, b, s.k, s.p, s.m, s.u);
    return;
  }

  // the cut
  uint64_t cut = (uint64_t)(DEAD + 1) << 32;
  if (listed) {
    if (s.by_count || n <= THREADS / 4 || !(s.p < 1.0f)) {
#pragma unroll
      for (int i = 0; i < CAP / THREADS; ++i)
        if (i * THREADS + t < n) S.list[i * THREADS + t] = member[i];
      __syncthreads();
      sort_list<true>(S, n);
    }
  }
  if (s.by_count) {
    const int few = min(n, s.k);   // (up to 1024: a token a thread)
    const uint64_t at = t < few ? S.list[t] : 0;
    const double w = t < few ? row.weight((uint32_t)(at >> 32)) : 0.0;
    double sum;
    const double before = group_scan(w, S.wave_f, &sum) - w;
    const bool stays = t < few && (t == 0 || ((!(s.p < 1.0f) || before < (double)s.p * sum) && !(w < (double)s.m)));
    const int left = __syncthreads_count(stays);
    cut = S.list[left - 1];
    __syncthreads();
    // in order of the index
    if (t < left) S.list[t] = ~((uint64_t)(uint32_t)~(uint32_t)at << 32 | (uint32_t)(at >> 32));
    __syncthreads();
    sort_list<false>(S, left);
    const uint64_t x = t < left ? ~S.list[t] : 0;
    const double y = t < left ? row.weight((uint32_t)x) : 0.0;
    const double upto = group_scan(y, S.wave_f, &sum);
    if (t == 0) S.found = left - 1;
    __syncthreads();
    first_thread(&S.found, t < left && upto > s.u * sum);
    __syncthreads();
    if (t == S.found) P.tokens[b] = (int)(x >> 32);
    if (t == 0) R.kind = BY_CUT, R.cut = cut, R.sum = sum;
    return;
  }

  place_chunk(s, chunk_best, top, t < P.chunks, G);
  const int lo = listed ? r.lo : BINS;
  // The list's share of every chunk.  min_p alone lets tokens of any weight stay, and what they have below 2^-LIST_BITS is added up by
  // itself, in multiples of 2^(-2 LIST_BITS) and no less than one; with top_p they weigh 2^-46 of the largest and more (one of less
  // and all behind it would be less than 2^-24 of the row).
  uint64_t* rest = reinterpret_cast<uint64_t*>(S.part);
  const bool any_weight = !(s.p < 1.0f);
  S.mass[t] = 0, rest[t] = 0;
  __syncthreads();
  if (listed) {
    double above = r.above;
    const double target = (double)s.p * r.total;
    bool from_top = lo == 0;
    if (n > THREADS / 4 && s.p < 1.0f) {
      // a long list: once more in bins, of its numbers' bits, and only the bin with the cut is sorted
      uint64_t* bins = reinterpret_cast<uint64_t*>(S.part);
      uint32_t most = 0, least = 0xffffffffu;
#pragma unroll
      for (int i = 0; i < CAP / THREADS; ++i)
        if (i * THREADS + t < n) most = max(most, (uint32_t)(member[i] >> 32)), least = min(least, (uint32_t)(member[i] >> 32));
      bins[t] = 0;
      const uint64_t ends = group_max_halves(most, ~least, S.wave64);
      most = (uint32_t)(ends >> 32), least = ~(uint32_t)ends;
      const int shift = max(32 - __builtin_clz((most - least) | 1) - 10, 0);   // (1024 bins)
      if (t == 0) S.n = 0, S.found = (most - least) >> shift;   // (if rounding lets none reach the target: the last)
      uint64_t w[CAP / THREADS];
#pragma unroll
      for (int i = 0; i < CAP / THREADS; ++i) {
        w[i] = 0;
        if (i * THREADS + t >= n) continue;
        const uint32_t key = (uint32_t)(member[i] >> 32);
        w[i] = whole_of(row.weight(key) * (double)(1ull << LIST_BITS));
        atomicAdd(reinterpret_cast<unsigned long long*>(&bins[(most - key) >> shift]), (unsigned long long)w[i]);
      }
      __syncthreads();
      uint64_t all;
      const uint64_t here = bins[t], upto = group_scan(here, S.wave64, &all);
      first_thread(&S.found, here > 0 && above + (double)upto / (double)(1ull << LIST_BITS) >= target);
      __syncthreads();
      const int bin = S.found;
      if (t == bin) S.hit = upto - here;
#pragma unroll
      for (int i = 0; i < CAP / THREADS; ++i) {
        if (i * THREADS + t >= n) continue;
        const uint32_t key = (uint32_t)(member[i] >> 32);
        const int at = (most - key) >> shift;
        if (at == bin)
          S.list[atomicAdd(&S.n, 1u)] = member[i];
        else if (at < bin && !(row.weight(key) < (double)s.m))
          atomicAdd(reinterpret_cast<unsigned long long*>(&S.mass[(int)~(uint32_t)member[i] / P.chunk]), (unsigned long long)w[i]);
      }
      __syncthreads();
      above += (double)S.hit / (double)(1ull << LIST_BITS);
      from_top = from_top && bin == 0;
      n = (int)S.n;
      sort_list<true>(S, n);
    }
    cut = n > 0 ? S.list[0] + 1 : cut;   // (none of the list)
    for (int i0 = 0; i0 < n; i0 += THREADS) {
      const int i = i0 + t;
      const uint64_t at = i < n ? S.list[i] : 0;
      const double w = i < n ? row.weight((uint32_t)(at >> 32)) : 0.0;
      double here;
      const double before = above + group_scan(w, S.wave_f, &here) - w;
      const bool stays = i < n && ((from_top && i == 0) || ((!(s.p < 1.0f) || before < target) && !(w < (double)s.m)));
      const int left = __syncthreads_count(stays);   // (the first so many: weights fall)
      if (left) cut = S.list[i0 + left - 1];
      if (stays) {
        const int c = (int)~(uint32_t)at / P.chunk;
        const double x = w * (double)(1ull << LIST_BITS), whole = any_weight ? floor(x) : x;
        atomicAdd(reinterpret_cast<unsigned long long*>(&S.mass[c]), (unsigned long long)whole_of(whole));
        if (any_weight)
          atomicAdd(reinterpret_cast<unsigned long long*>(&rest[c]), (unsigned long long)whole_of(ceil((x - whole) * (double)(1ull << LIST_BITS))));
      }
      above += here;
    }
    __syncthreads();
  }
  // the chunk
  const double share = t >= P.chunks ? 0.0
                       : (lo == 0 ? 0.0 : chunk_upto(P, G, (int64_t)b * P.chunks, t, lo - 1)) +
                             ((double)S.mass[t] + (any_weight ? (double)rest[t] / (double)(1ull << LIST_BITS) : 0.0)) / (double)(1ull << LIST_BITS);
  double sum;
  const double upto = group_scan(share, S.wave_f, &sum);
  const double target = s.u * sum;
  if (t == 0) S.found = P.chunks, S.n = 0;
  __syncthreads();
  first_thread(&S.found, share > 0.0 && upto > target);
  last_thread(&S.n, share > 0.0);
  __syncthreads();
  const int c = S.found < P.chunks ? S.found : (int)S.n;   // (if rounding lets none pass: the last with any weight)
  if (t == c) S.hit = __builtin_bit_cast(uint64_t, upto - share);
  if (t == 0) R.kind = BY_CUT, R.cut = cut, R.sum = sum;
  __syncthreads();
  // the token: a wave takes a part of the chunk in one piece, 64 logits at a time
  const int lane = t & 63, wave = t >> 6, i0 = c * (PER * THREADS) + wave * (PER * 64) + lane;
  uint32_t key[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) key[e] = row.key(min(i0 + e * 64, V - 1));
#pragma unroll
  for (int e = 0; e < PER; ++e) key[e] = i0 + e * 64 < V ? key[e] : 0;
  double w[PER], part = 0.0;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const bool stays = key[e] > DEAD && place_of(key[e], i0 + e * 64) >= cut;
    w[e] = row.weight(max(key[e], DEAD + 1));
    if (!stays || w[e] < (double)s.m) w[e] = 0.0;   // (min_p: an empty list has no cut)
    part += w[e];
  }
  double all;
  group_scan(part, S.wave_f, &all);
  double before = __builtin_bit_cast(double, S.hit);
  int in = -1, some = -1;   // the wave the token is in; the last with any weight
  for (int v = 0; v < WAVES; ++v) {
    if (!(S.wave_f[v] > 0.0)) continue;
    some = v;
    if (in < 0 && before + S.wave_f[v] > target) in = v;
    if (in < 0) before += S.wave_f[v];
  }
  const bool passed = in >= 0;
  if (wave != (passed ? in : some)) return;
  int token = -1, last = 0;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const double here = wave_scan(w[e]);
    const uint64_t past = __ballot(passed && w[e] > 0.0 && before + here > target), any = __ballot(w[e] > 0.0);
    if (any) last = i0 - lane + e * 64 + 63 - __builtin_clzll(any);
    if (past && token < 0) token = i0 - lane + e * 64 + __builtin_ctzll(past);
    before += of_last_lane(here);
  }
  if (lane == 0) P.tokens[b] = token < 0 ? last : token;
}

template <typename E, int PER> __global__ __launch_bounds__(THREADS, 8) void oscar_sample_probs_kernel(SampleParams P) {
  __shared__ uint64_t s_wave[WAVES];
  __shared__ double s_power[32];
  const int b = blockIdx.y, c = blockIdx.x, t = threadIdx.x;
  float x[PER];
  load_row<E, PER>(P, b, c, x);
  const uint64_t chunk_best = t < P.chunks ? P.best[(int64_t)b * P.chunks + t] : 0;
  const Settings s = settings(P, b);
  const RowState R = P.rows[b];
  const int kind = R.kind;
  if (kind == DONE) return;
  fill_powers(s_power);
  const uint64_t best = group_max(chunk_best, s_wave);
  const double top = (double)number_of((uint32_t)(best >> 32)), scale = 1.4426950408889634 / (double)s.temp;
  // (of nothing: NaN, which no logit reaches)
  const uint64_t cut = kind == BY_CUT ? R.cut : kind == ONE_TOKEN ? best : ~0ull;
  const float cut_x = number_of((uint32_t)(cut >> 32));
  const uint32_t cut_i = ~(uint32_t)cut;
  const double inv_sum = kind == BY_CUT ? 1.0 / R.sum : 1.0;
  float* out = P.probs + (int64_t)b * P.V;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int i = c * (PER * THREADS) + e * THREADS + t;
    if (i >= P.V) break;
    float y = 0.0f;
    if (x[e] > cut_x || (x[e] == cut_x && (uint32_t)i <= cut_i)) {
      const double w = power_of_2<0>(((double)x[e] - top) * scale, s_power);
      y = kind == ONE_TOKEN ? 1.0f : w < (double)s.m ? 0.0f : (float)(w * inv_sum);
    }
    __builtin_nontemporal_store(y, out + i);
  }
}

// Logits of a chunk: 4096 as long as a CU has no second one, else 8192 (top_p over 32 rows of 32000: 32.3 us in pieces of
// 4096, 33.8 in pieces of 8192; 64: 36.6 and 34.7; 16 of 128003: 45 and 38; 64: 78 and 59).
int chunk_of(int32_t batch, int32_t vocab) { return (int64_t)batch * ((vocab + 4095) / 4096) <= 256 ? 4096 : 8192; }

template <typename E, int PER> void launch(const SampleParams& P, int batch, hipStream_t st) {
  const dim3 grid(P.chunks, batch);
  hipLaunchKernelGGL((oscar_sample_bins_kernel<E, PER>), grid, dim3(THREADS), 0, st, P);
  if (P.top_k || P.top_p || P.min_p) {
    // Each chunk for itself, or a launch for the bins: a draw takes 23.1 and 24.6 us of one row of 32000, 30.2 and 31.3 of
    // 16 (128 chunks), 32.7 and 32.3 of 32, 68 and 59 of 64 of 128003
    // (pieces of 8192 are 129 and more)
    if (PER == 4 && (int64_t)P.chunks * batch <= 128) {
      hipLaunchKernelGGL((oscar_sample_list_kernel<E, 4, true>), grid, dim3(THREADS), 0, st, P);
    } else {
      hipLaunchKernelGGL(oscar_sample_find_kernel, dim3(batch), dim3(THREADS), 0, st, P);
      hipLaunchKernelGGL((oscar_sample_list_kernel<E, PER, false>), grid, dim3(THREADS), 0, st, P);
    }
  }
  hipLaunchKernelGGL((oscar_sample_pick_kernel<E, PER>), dim3(batch), dim3(THREADS), 0, st, P);
  if (P.probs) hipLaunchKernelGGL((oscar_sample_probs_kernel<E, PER>), grid, dim3(THREADS), 0, st, P);
}
template <typename E> void launch(const SampleParams& P, int batch, hipStream_t st) {
  P.chunk == 4096 ? launch<E, 4>(P, batch, st) : launch<E, 8>(P, batch, st);
}

}  // namespace

extern "C" size_t oscar_sample_workspace_bytes(int32_t batch, int32_t vocab) {
  if (batch < 1 || batch > 65535 || vocab < 1 || vocab > OSCAR_SAMPLE_MAX_VOCAB) return 0;
  const size_t chunk = chunk_of(batch, vocab), chunks = (vocab + chunk - 1) / chunk;
  return batch * (chunks * (BINS + 1) * sizeof(uint64_t) + sizeof(RowState) + CAP * sizeof(uint64_t));
}

extern "C" int oscar_sample(const void* logits, int64_t row_stride, int32_t batch, int32_t vocab, int32_t dtype,
                            const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                            const float* u, int32_t* tokens, float* probs, void* workspace, size_t workspace_bytes,
                            void* stream) {
  if (dtype != OSCAR_F32 && dtype != OSCAR_BF16 && dtype != OSCAR_F16) return OSCAR_ERR_INVALID_ARG;
  if (batch < 0 || batch > 65535 || vocab < 1 || vocab > OSCAR_SAMPLE_MAX_VOCAB || (batch > 1 && row_stride < vocab))
    return OSCAR_ERR_INVALID_ARG;
  if (batch == 0) return OSCAR_OK;
  if (!logits || !u || !tokens) return OSCAR_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == OSCAR_F32 ? 4 : 2) != 0) return OSCAR_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < oscar_sample_workspace_bytes(batch, vocab) || (reinterpret_cast<uintptr_t>(workspace) & 15) != 0)
    return OSCAR_ERR_WORKSPACE;
  SampleParams P = {};
  P.logits = logits;
  P.stride = row_stride;
  P.V = vocab;
  P.chunk = chunk_of(batch, vocab);
  P.chunks = (vocab + P.chunk - 1) / P.chunk;
  P.temperature = temperature;
  P.top_p = top_p;
  P.min_p = min_p;
  P.u = u;
  P.top_k = top_k;
  P.tokens = tokens;
  P.probs = probs;
  P.best = reinterpret_cast<uint64_t*>(workspace);
  P.cum = P.best + (size_t)batch * P.chunks;
  P.list = P.cum + (size_t)batch * P.chunks * BINS;
  P.rows = reinterpret_cast<RowState*>(P.list + (size_t)batch * CAP);
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
