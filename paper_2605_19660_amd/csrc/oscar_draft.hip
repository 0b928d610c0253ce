// oscar_draft_attn: attention of several new tokens of every sequence over its packed cache and, causally,
// over each other.
//
//   logit[t][h][i] = scale n_i sum_j Q_j (Delta_k c_k - Delta_k z_k)_ij   cached token i, Q = H(q_th)/sqrt(128)
//                                                                        (float zero-points: Delta_k c_k + zero)
//   logit[t][h][j] = scale <q_th, k_j>                                   new token j <= t
//   out[t][h]      = softmax over both, times the values
//
// The T tokens' g query heads of a kv head are T g rows that read the same keys and values.  A wave holds 16 or
// 32 of them (16 a matrix tile) and takes whole pages of 128 tokens on its own, with its own running state, so
// that nothing in the page loop waits for another wave; the four waves of a workgroup and the splits of the
// sequence are joined at the end.
//   S^T = K Q^T  : v_mfma_f32_16x16x32_f16, rows = 16 tokens, columns = 16 query rows, over 128 channels
//   O^T = V^T P^T: rows = 16 channels, columns = query rows, over 128 tokens
// Row n of a token tile is token 4 (n % 4) + n / 4 of it: a lane's four results of tile T are then its tokens
// 16 T + 4 r + lane / 16, exactly those whose value codes the lane's chunk of the page holds for k-step r: the
// probabilities are packed where they are and become operands without an exchange.
// (Four waves on one page, a quarter of its tokens and of its channels each, probabilities through LDS: 2.3 times
// the LDS traffic, 1.4 times the matrix products and a barrier a page; with one limb an operand, see below, 8 new tokens
// over 8 x 32K took 99 us so and 73 as it is.)
//
// Codes become fp16 operands with a mask (a code parked in the mantissa of a subnormal: c 2^(s - 24)); the
// steps go to the other operand, Q Delta_k and P Delta_v, and 2^-s with them.  As in the decode kernels that operand is
// carried in two fp16 limbs, hi + lo, each a matrix product of its own: 22 bits.  The limbs come out of packed fp16
// arithmetic on a multiplicand split once (times()).  The zero terms are products on the matrix cores too, in limbs
// themselves: for the keys what a tile's sums start from, for the values one extra tile, whose other rows are the rows'
// sums.  With one limb, half a step (2^-11) each for Q, Q Delta, P, P Delta and the zero terms, fp16 outputs were off by
// 4e-4 .. 3e-3 of their length, where their own rounding is 2e-4; the second limb costs 1.2 .. 1.55 times the time.
// Everything that meets a limb is first brought to fp16's middle by powers of two, in both directions, and the fp32 sums
// carry the exponents: a query by its largest channel, a page's key steps and zero terms by its largest,
// its value steps and zero terms by the largest of their value group so far.  The probabilities are stored below 2^15.
// So a product keeps its 22 bits down to 2^-28 of the largest the group can have, and a step its own 11 down to 2^-14 of
// the largest step; an unscaled P Delta lost 0.3 .. 15 % of what values of 1e-2 .. 3e-4 add beside a token that takes the
// softmax without values.  16-bit values of the window and of new tokens: fp16 ones as they are, bf16 ones as bf16
// against probabilities of two bf16 limbs, so that they keep their range.  Sums, maxima and outputs are fp32.
//
// What bounds it: the issue of instructions.  A page costs a wave with two tiles 304 matrix and about 1250 vector
// instructions, and the two hardly overlap across the waves of a SIMD (matrix cores busy 40 % of the time, other vector
// instructions being issued 52 %).  8 new tokens of 32 heads over 8 x 32768: 95 us, 1.9 TB/s, and 5 in the reduce pass; 5
// of 28 heads over 131001, G_k = 32: 53 + 5; 500 of 32 heads over two caches of 8100, 4-bit: 324 us, 420 TFLOP/s of the
// products that the formula has; 4 over 1000: 11 + 4, a chain of lengths, page, window and reduce pass.
// Registers: two workgroups a CU leave a wave 256.  Two tiles with 4-bit codes, fp32 metadata or k_group below 128 keep
// 5 .. 62 of theirs in scratch memory (up to 21 accesses a page), all other variants none.
#include "oscar_decode_common.h"

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// (said to be in device memory: through pointers of which the compiler does not know that, loads are counted with
// those of LDS and every wait for one is a wait for all)
typedef const __attribute__((address_space(1))) uint8_t* DevicePtr;
template <typename T> __device__ __forceinline__ T load_as(DevicePtr p) {
  return *reinterpret_cast<const __attribute__((address_space(1))) T*>(p);
}

constexpr float kHalfMax = 65504.0f;
constexpr float kBf16Most = 1152921504606846976.0f;   // 2^60: bf16 values beyond it count as that
constexpr int kQTop = 14;            // a query's largest channel is scaled to below 2^14

// What loads of a page that is none take: its codes and parameters are zeros, and nothing that follows is NaN.
__device__ __align__(256) const uint8_t kNoPage[8192] = {};

// Division of n < 2^31 by a number known on the host (as a division it is 20 instructions, one after the other).
struct Divisor {
  uint32_t d, m;   // m = (2^32 - 1) / d: the product falls short by less than one
  __device__ __forceinline__ int of(int n) const {
    const uint32_t q = __umulhi((uint32_t)n, m);
    return (int)(q + ((q + 1) * d <= (uint32_t)n ? 1 : 0));
  }
};
Divisor divisor(int d) { return {(uint32_t)d, 0xffffffffu / (uint32_t)d}; }

struct DraftParams {
  const void *q, *k_new, *v_new;
  void* out;
  float* ws;
  const int32_t* new_lens;
  oscar_cache c;
  PageGeom g;
  int T, num_splits, group;   // group: query heads of a kv head
  bool last_first;            // order of the blocks of rows
  Divisor by_splits, by_kv_heads, by_group, by_step;   // by_step: the waves of all splits
  float scale_log2;
};

template <int BITS> struct Codes {
  static constexpr int BPMIN = BITS == 2 ? 4 : 2;
  // the operand of k-step kk from a chunk
  __device__ static __forceinline__ half8 operand(const uint32_t* w, int kk) {
    u32x4 r;
    if (BITS == 2) {
      const uint32_t x = w[kk / 2];
      if (kk % 2 == 0) {
        const uint32_t l = x << 4;
        r[0] = l & 0x00300030u, r[1] = l & 0x00C000C0u, r[2] = x & 0x00300030u, r[3] = x & 0x00C000C0u;
      } else {
        const uint32_t l = x >> 6;
        r[0] = x & 0x03000300u, r[1] = l & 0x00300030u, r[2] = l & 0x00C000C0u, r[3] = l & 0x03000300u;
      }
    } else {
      const uint32_t x = w[kk], l = x << 2, s = x >> 6;
      r[0] = l & 0x003C003Cu, r[1] = l & 0x03C003C0u, r[2] = s & 0x003C003Cu, r[3] = s & 0x03C003C0u;
    }
    return __builtin_bit_cast(half8, r);
  }
  // what an element's bit position is above the lowest
  __host__ __device__ static constexpr int above(int kk, int e) { return slot_bitpos(BITS, kk, e) - BPMIN; }
  // 2^above, the other operand's counterweight for what is no code (kk counts modulo 2)
  __device__ static __forceinline__ half8 counterweight(int kk) {
    half8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (_Float16)(float)(1 << above(kk, e));
    return r;
  }
};

// A number in two fp16 limbs: 22 bits of it, while its low limb stays above the smallest fp16 number.
struct Limbs {
  half8 hi, lo;
};
__device__ __forceinline__ half8 fma8(half8 a, half8 b, half8 c) { return __builtin_elementwise_fma(a, b, c); }
// The product of two numbers in limbs: of the high limbs its high limb and the rest, which fp16 holds exactly, and the
// products of a high and a low limb.  FINE: the factor has a low limb (fp16 steps have none).
template <bool FINE> __device__ __forceinline__ Limbs times(half8 hi, half8 lo, const half8* by) {
  const half8 h = hi * by[0];
  half8 rest = fma8(lo, by[0], fma8(hi, by[0], -h));
  if (FINE) rest = fma8(hi, by[1], rest);
  return {h, rest};
}

// A page's metadata as the waves read it: steps and zero terms (with their counterweights, in two limbs) as fp16 in
// operand order, norms as fp32 with the keys' exponent.
template <bool M32> struct Staged {
  static constexpr int LIMBS = M32 ? 2 : 1;   // of a step
  half8 k_step[LIMBS][64], k_zero[2][64];   // [limb][group][quarter][k-step]
  half8 v_step[LIMBS][64], v_zero[2][80];   // [limb][group][k-step][quarter]; behind the four groups the counterweights alone
  float norm[R];                            // position (token % 16) * 8 + token / 16
};
// A row's probabilities are taken against a reference that follows its maximum only when that has passed it by
// 2^kSlack: over long sequences the maximum creeps up in many small steps, and each costs a rescaling of the
// whole state (8 new tokens over 8 x 32K: 102 us, 108 with a reference that follows at once).
constexpr float kSlack = 8.0f, kNone = -3e38f;
constexpr int kOff = 7;          // exponent of a probability at its reference: kOff + kSlack stay inside fp16
__device__ __forceinline__ float exp2i(int x) { return __uint_as_float((uint32_t)(127 + x) << 23); }   // |x| < 127
// What a lane holds of the metadata of a page to come: 8 steps and 8 zeros of the keys or of the values.
template <bool M32> struct Fetched {
  u32x4 a[M32 ? 2 : 1], b[M32 ? 2 : 1];
  __device__ __forceinline__ void load(DevicePtr src, DevicePtr zsrc, uint32_t at) {
#pragma unroll
    for (int i = 0; i < (M32 ? 2 : 1); ++i) {
      a[i] = load_as<u32x4>(src + at + 16 * i);
      b[i] = load_as<u32x4>(zsrc + at + 16 * i);
    }
  }
  __device__ __forceinline__ static float number(const u32x4* x, int e) {
    if (M32) return __uint_as_float(x[e / 4][e % 4]);
    return (float)__builtin_bit_cast(half8, x[0])[e];
  }
  // x with all eight steps below 2^x (within its limits) and all zero terms below 2^(x + 11): times 2^-x, and with their
  // counterweights (2^4 at most), fp16 holds them.
  __device__ __forceinline__ int exponent(float ints) const {
    if (M32) {
      float s = 0.0f, t = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s = fmaxf(s, number(a, e));
        t = fmaxf(t, fabsf(zero_term(ints, number(a, e), number(b, e))));
      }
      return min(max(max((int)(__float_as_uint(s) >> 23), (int)(__float_as_uint(t) >> 23) - 11) - 126, -40), 100);
    }
    // fp16 bits as logarithms: those of a product are the factors' added, and one more at most
    const bool whole = ints != 0.0f;
    const uint32_t with = whole ? 0xffffffffu : 0u, less = whole ? 0x64006400u : 0x2c002c00u;   // 25 and 11 in the exponent
    ushort2v most = {0, 0};
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const uint32_t st = a[0][d], z = b[0][d] & 0x7fff7fffu, s = st & with;   // (a bit cast of a vector's element takes its first)
      most = __builtin_elementwise_max(most, __builtin_bit_cast(ushort2v, st));
      most = __builtin_elementwise_max(most, __builtin_elementwise_sub_sat(__builtin_bit_cast(ushort2v, z) + __builtin_bit_cast(ushort2v, s),
                                                                           __builtin_bit_cast(ushort2v, less)));
    }
    return (max((int)most[0], (int)most[1]) >> 10) - 14;
  }
  __device__ __forceinline__ static float zero_term(float ints, float s, float z) { return z * (ints != 0.0f ? -s : 1.0f); }
  // Step and zero term times 2^-x; a number is step c + zero: zero = -step z for integer zero-points (ints = 1), z itself
  // for float ones (ints = 0), as one form: nothing here branches.
  __device__ __forceinline__ void step_and_zero(float ints, int x, Limbs& step, Limbs& zero) const {
    const float by = exp2i(-x);
    if (M32) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float s = number(a, e), z = number(b, e);
        const float t = __builtin_amdgcn_fmed3f(zero_term(ints, s, z) * by, -kHalfMax, kHalfMax);   // (infinite ones)
        const float u = fminf(s * by, kHalfMax);
        step.hi[e] = (_Float16)u;
        step.lo[e] = (_Float16)(u - (float)step.hi[e]);
        zero.hi[e] = (_Float16)t;
        zero.lo[e] = (_Float16)(t - (float)zero.hi[e]);
      }
    } else {
      const half8 z = __builtin_bit_cast(half8, b[0]);
      // (registers: as constants or halves of one they are taken apart into single operations)
      uint32_t two[3] = {__builtin_bit_cast(uint32_t, (half2v)(_Float16)by),
                         __builtin_bit_cast(uint32_t, (half2v)(_Float16)ints),
                         __builtin_bit_cast(uint32_t, (half2v)(_Float16)(ints != 0.0f ? -1.0f : by))};
      asm("" : "+v"(two[0]), "+v"(two[1]), "+v"(two[2]));
      auto splat = [](uint32_t w) { return __builtin_bit_cast(half8, (u32x4){w, w, w, w}); };
      const half8 one = (_Float16)1.0f;
      step.hi = __builtin_bit_cast(half8, a[0]) * splat(two[0]);
      const half8 f = fma8(step.hi, splat(two[1]), one - splat(two[1])), m = z * splat(two[2]);   // step or 1, -z or z 2^-x
      zero.hi = f * m;
      zero.lo = fma8(f, m, -zero.hi);
    }
  }
};

__device__ __forceinline__ float4v mfma(half8 a, half8 b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float4v mfma(bf16x8 a, bf16x8 b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// The largest of the 16 lanes of a row, in all of them.
template <int CTRL> __device__ __forceinline__ int row_max_step(int v) {
  return max(v, __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ int row16_max(int v) {
  v = row_max_step<0x128>(v);   // row_ror:8, 4, 2, 1
  v = row_max_step<0x124>(v);
  v = row_max_step<0x122>(v);
  return row_max_step<0x121>(v);
}
__device__ __forceinline__ int max_of_rows(int v) {   // over the four rows
  auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max((int)a[0], (int)a[1]);
  a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max((int)a[0], (int)a[1]);
}
__device__ __forceinline__ half2v pack2(float a, float b) { return __builtin_convertvector((float2v){a, b}, half2v); }
// Two numbers into limbs, as elements e and e + 1 (constants where this is used).  (The rests as products with a
// register of -1: mixed operations take the fp16 numbers as they are, subtractions widen them first.)
__device__ __forceinline__ void split2(float a, float b, Limbs& x, int e) {
  float less = -1.0f;
  asm("" : "+s"(less));
  const half2v hi = pack2(a, b), lo = pack2(fmaf((float)hi[0], less, a), fmaf((float)hi[1], less, b));
  x.hi[e] = hi[0], x.hi[e + 1] = hi[1];
  x.lo[e] = lo[0], x.lo[e + 1] = lo[1];
}
__device__ __forceinline__ float max_of_row(float v) {   // over the four lanes that hold a query row
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

constexpr int TAIL = 32;         // tokens of a 16-bit piece (window, new tokens)

constexpr int OROW = D + 4;
template <int NR, bool M32> struct Lds {
  static constexpr int ROWS = NR * 16;
  struct Loop {
    u32x4 q[NR][4][64];                              // queries as they came,
    half8 qh[NR][2][4][64], qc[NR][2][4][64];        // rotated and scaled, in limbs, and in the codes' order
    half8 cw[2];                                     // counterweights of even and odd k-steps
    float unit[NR][16];                              // of a row's scaled query
    union {
      Staged<M32> meta;                              // of a wave's page,
      half8 tail[TAIL][9];                           // of its 16-bit piece: half of its values' channels
    } of_wave[4];
  };
  struct Join {
    float o[4][ROWS][OROW], m[4][ROWS], l[4][ROWS];
  };
  union {
    Loop loop;
    Join join;
  };
  __device__ Lds() {}
};

// ONE: k_group is the whole page.
template <int BITS, bool M32, bool ONE, int NR>
__device__ __forceinline__ void attend(const DraftParams& P, Lds<NR, M32>& lds, int row0) {
  using C = Codes<BITS>;
  constexpr int ROWS = NR * 16;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, q4 = lane >> 4;
  const int Hkv = P.c.cfg.n_kv_heads, Hq = P.c.cfg.n_q_heads, g = P.group;
  const int unit = P.by_splits.of(blockIdx.x), split = blockIdx.x - unit * P.num_splits;
  const int b = P.by_kv_heads.of(unit), kvh = unit - b * Hkv;

  // the queries' loads wait for nothing
  const uint16_t* q_row[NR];
  int row_t[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const int row = min(row0 + 16 * i + n, P.T * g - 1);
    row_t[i] = P.by_group.of(row);
    q_row[i] = reinterpret_cast<const uint16_t*>(P.q) +
               (((size_t)b * P.T + row_t[i]) * Hq + (size_t)kvh * g + (row - row_t[i] * g)) * D + 32 * q4;
  }
  u32x4 q_in[4];
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) q_in[kk] = *reinterpret_cast<const u32x4*>((wave == 0 ? q_row[0] : q_row[NR - 1]) + 8 * kk);

  // ---- what this wave takes: pages, then 16-bit pieces (window, then new tokens), dealt to the waves of all splits ----
  // (the first pages are known ahead of the lengths, so that their table entries are read together with those; the
  // table as constant memory, by the scalar unit: a vector load's wait would be one for every load ahead)
  const int step = P.num_splits * 4, own = split * 4 + wave;
  const auto table = reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(
      reinterpret_cast<uintptr_t>(P.c.block_table + (size_t)b * P.c.max_pages_per_seq));
  auto entry_of = [&](int p) { return table[min(p, P.c.max_pages_per_seq - 1)]; };
  const int entry0 = entry_of(own), entry1 = entry_of(own + step);
  const int n_new = P.new_lens ? min(max(P.new_lens[b], 0), P.T) : P.T;
  const int seq_len = max(P.c.seq_lens[b], 0);
  const int res = min(max(P.c.res_lens[b], 0), min(R, seq_len));
  const int pages = min((seq_len - res) / R, P.c.max_pages_per_seq);
  const int rows = min(max(n_new * g - row0, 0), ROWS);         // of this block that are there
  const float ints = P.c.cfg.zp_mode == OSCAR_ZP_MIN ? 0.0f : 1.0f;
  const bool bf16 = P.c.cfg.io_dtype == OSCAR_BF16;

  float4v o[NR][8];   // channels 16 ct + 4 q4 + r of row n, in units of the codes once pages have begun
  float4v x[NR];      // row 4 q4 + r of the extra tile: 0 .. 3 the value groups' mean terms, 4 the row's sum
  float M[NR];        // the row's reference, log2 units, less the exponent kOff its probability has there
  float most[NR];     // how far a logit may be above M; kNone before the row's first token
#pragma unroll
  for (int i = 0; i < NR; ++i) {
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) o[i][ct] = (float4v){0, 0, 0, 0};
    x[i] = (float4v){0, 0, 0, 0};
    M[i] = 0.0f;
    most[i] = kNone;
  }

  if (rows > 0) {
    const int last_t = P.by_group.of(row0 + rows - 1);                   // last new token any row here sees
    const int n_win = (res + TAIL - 1) / TAIL;
    const int n_tail = n_win + (min(n_new, last_t + 1) + TAIL - 1) / TAIL;
    int piece = own - (pages - P.by_step.of(pages) * step);
    piece += piece < 0 ? step : 0;
    int page = own;
    // What is no page (past the end, or not of the pools) takes the zeros: every iteration makes the same loads.
    struct Page {
      int phys;
      bool held;
    };
    auto page_of = [&](int p, int phys) { return Page{phys, p < pages && phys >= 0 && phys < P.c.num_pages}; };

    // ---- loads ahead ----
    // (a page ahead; of two tiles the keys' codes and the metadata go out halfway through the values, and 4-bit values'
    // codes by halves: the registers do not hold more.  8 new tokens over 8 x 32K 97 us, 103 with the keys' codes ahead of
    // all values and spilled; 4-bit 117 and 138)
    constexpr int AHEAD = BITS == 4 && NR == 2 ? 2 : 4;
    constexpr bool LATE = NR == 2;
    uint32_t kc[4][2 * BITS], vc[4][2 * BITS];
    // (every part of a page has a power of two of bytes)
    constexpr int code_shift = BITS == 2 ? 12 : 13, norm_shift = M32 ? 9 : 8;
    const int k_shift = norm_shift + 1 + (ONE ? 0 : P.g.ngk >> 1), v_shift = norm_shift + 1 + (P.g.ngv >> 1);
    auto pool_of = [&](const void* pool, int shift, const Page& pg) {
      const uintptr_t at = reinterpret_cast<uintptr_t>(pool) + (((size_t)pg.phys * Hkv + kvh) << shift);
      return reinterpret_cast<DevicePtr>(pg.held ? at : reinterpret_cast<uintptr_t>(kNoPage));
    };
    const uint32_t k_at = chunk_offset(BITS, 0, 4 * (n % 4) + n / 4, q4), v_at = chunk_offset(BITS, 0, n, q4);
    auto load_codes = [&](DevicePtr page, uint32_t at, uint32_t (&w)[4][2 * BITS], int first, int end) {
#pragma unroll
      for (int c = first; c < end; ++c)
#pragma unroll
        for (int j = 0; j < BITS / 2; ++j)
          *reinterpret_cast<u32x4*>(&w[c][4 * j]) = load_as<u32x4>(page + at + chunk_offset(BITS, 2 * c, 0, 0) + 16 * j);
    };
    constexpr int MB = M32 ? 4 : 2;
    const uint32_t km_at = (uint32_t)min(lane, 16 * P.g.ngk - 1) * 8 * MB, vm_at = (uint32_t)min(lane, 16 * P.g.ngv - 1) * 8 * MB;
    Fetched<M32> fk, fv;
    u32x4 fn;
    auto fetch_meta = [&](const Page& pg) {
      const DevicePtr km = pool_of(P.c.k_meta, k_shift, pg);
      const DevicePtr vm = pool_of(P.c.v_meta, v_shift, pg);
      fk.load(km, km + (1 << k_shift >> 1), km_at);
      fv.load(vm, vm + (1 << v_shift >> 1), vm_at);
      const DevicePtr kn = pool_of(P.c.k_norms, norm_shift, pg);
      if (M32) {
        fn[0] = load_as<uint32_t>(kn + lane * 8), fn[1] = load_as<uint32_t>(kn + lane * 8 + 4);
      } else {
        fn[0] = load_as<uint32_t>(kn + lane * 4);
      }
    };
    Staged<M32>& meta = lds.loop.of_wave[wave].meta;
    auto stage_keys = [&] {
      Limbs st, zero;
      const int x_keys = max_of_rows(row16_max(fk.exponent(ints)));   // of the page
      fk.step_and_zero(ints, x_keys, st, zero);
      const float unit = exp2i(x_keys);
      const half8 cw = lds.loop.cw[lane % 2];
      meta.k_step[0][lane] = st.hi;
      if (M32) meta.k_step[M32 ? 1 : 0][lane] = st.lo;
      meta.k_zero[0][lane] = zero.hi * cw;
      meta.k_zero[1][lane] = zero.lo * cw;
      float v[2];
      if (M32) {
        v[0] = __uint_as_float(fn[0]), v[1] = __uint_as_float(fn[1]);
      } else {
        const half2v h = __builtin_bit_cast(half2v, fn[0]);
        v[0] = (float)h[0], v[1] = (float)h[1];
      }
      *reinterpret_cast<float2v*>(&meta.norm[2 * lane]) = (float2v){v[0] * unit, v[1] * unit};
    };
    // Values are summed in units of 2^x, x the lane's value group's largest exponent so far (of lane / 16).
    auto stage_values = [&](int x_before) {
      Limbs st, zero;
      const int x_now = max(x_before, row16_max(fv.exponent(ints)));
      fv.step_and_zero(ints, x_now, st, zero);
      const half8 cw = lds.loop.cw[lane / 4 % 2];
      meta.v_step[0][lane] = st.hi;
      if (M32) meta.v_step[M32 ? 1 : 0][lane] = st.lo;
      meta.v_zero[0][lane] = zero.hi * cw;
      meta.v_zero[1][lane] = zero.lo * cw;
      return x_now;
    };

    Page pg0 = page_of(page, entry0), pg1 = page_of(page + step, entry1);
    fetch_meta(pg0);
    load_codes(pool_of(P.c.k_codes, code_shift, pg0), k_at, kc, 0, 4);
    load_codes(pool_of(P.c.v_codes, code_shift, pg0), v_at, vc, 0, AHEAD);

    // ---- queries ----
    // Wave i rotates tile i, on the matrix cores: out = H q, H's signs exact in either type.  Row m of output tile
    // ot is channel 32 (m / 4) + 4 ot + m % 4, so that a lane ends with channels 32 q4 .. + 31 of its query row, as
    // the keys' operands have them; its input channels are 32 q4 + 8 kk + e.  The sign of H[i][j] is the parity of
    // i & j, taken apart into what depends on (n, e), on (ot, kk, e) and on (n, q4).
    if (wave < NR) {
      float y[8][4];   // channels 32 q4 + 4 ot + r
      float top_q = 0.0f;
      const bool there = row0 + 16 * wave + n < n_new * g;
      const bool rotate = P.c.cfg.rotation == OSCAR_ROTATION_ON;
      const float mul = P.scale_log2 * (rotate ? 0.08838834764831845f : 1.0f);
      const uint32_t one = bf16 ? 0x3f803f80u : 0x3c003c00u;
      // low two bits: e % 4 against n % 4; top two: q4 against n / 4
      u32x4 signs;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const uint32_t even = __popc((2 * d) % 4 & n), odd = __popc((2 * d + 1) % 4 & n), top = __popc(q4 & (n >> 2));
        signs[d] = one | (even + top) << 15 & 0x8000u | (odd + top) << 31;
      }
#pragma unroll
      for (int ot = 0; ot < 8; ++ot) {
        float4v acc = {0, 0, 0, 0};
        if (rotate) {
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            // bits 2 .. 4 of the input channel are 2 kk + e / 4 (8 kk + e below 32)
            const uint32_t lo = __popc(ot & 2 * kk) << 15 & 0x8000u, hi = __popc(ot & (2 * kk + 1)) << 15 & 0x8000u;
            const uint32_t flip[2] = {lo | lo << 16, hi | hi << 16};
            const u32x4 h = {signs[0] ^ flip[0], signs[1] ^ flip[0], signs[2] ^ flip[1], signs[3] ^ flip[1]};
            if (bf16)
              acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, h), __builtin_bit_cast(bf16x8, q_in[kk]),
                                                            acc, 0, 0, 0);
            else
              acc = mfma(__builtin_bit_cast(half8, h), __builtin_bit_cast(half8, q_in[kk]), acc);
          }
        } else {
          const u32x4 two = q_in[ot / 2];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const uint32_t v = two[(ot % 2) * 2 + r / 2] >> (16 * (r % 2)) & 0xffffu;
            acc[r] = bf16 ? __uint_as_float(v << 16) : __half2float(__ushort_as_half((uint16_t)v));
          }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          y[ot][r] = there ? acc[r] * mul : 0.0f;
          top_q = fmaxf(top_q, fabsf(y[ot][r]));
        }
      }
      // A query's scale, a power of two of its own: limbs then hold its largest products to 2^-22 and all others to 2^-38
      // of the largest.  (One for a block of rows would save a multiplication a logit, 2 %, and a query that is no number
      // would spoil the other rows of its block.)
      const int q_exp = min(max(kQTop - 1 + 127 - (int)(__float_as_uint(max_of_row(top_q)) >> 23), -100), 100);
      if (q4 == 0) lds.loop.unit[wave][n] = exp2i(-q_exp);
      const float by = exp2i(q_exp);
      Limbs qh[4];
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = y[2 * kk + e / 4][e % 4] * by;
          qh[kk].hi[e] = (_Float16)v;
          qh[kk].lo[e] = (_Float16)(v - (float)qh[kk].hi[e]);
        }
        lds.loop.q[wave][kk][lane] = q_in[kk];
        lds.loop.qh[wave][0][kk][lane] = qh[kk].hi;
        lds.loop.qh[wave][1][kk][lane] = qh[kk].lo;
      }
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        Limbs qc;   // in the codes' order, with the counterweights of their bit positions
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int u = slot_index(BITS, kk, e);
          const _Float16 w = (_Float16)(1.0f / (float)(1 << C::above(kk, e)));
          qc.hi[e] = qh[u / 8].hi[u % 8] * w;
          qc.lo[e] = qh[u / 8].lo[u % 8] * w;
        }
        lds.loop.qc[wave][0][kk][lane] = qc.hi;
        lds.loop.qc[wave][1][kk][lane] = qc.lo;
      }
    }
    // (constants of the page loop wait in LDS: the registers are spoken for)
    if (lane < 2) lds.loop.cw[lane] = lane == 0 ? C::counterweight(0) : C::counterweight(1);   // (the same from every wave)
    __syncthreads();
    float q_unit[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) q_unit[i] = lds.loop.unit[i][n];

    auto scale = [&](int i, float by) {
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) o[i][ct] *= by;
      x[i] *= by;
    };
    // New references for a tile one of whose rows has passed its own, and the state against them, in whole powers of two.
    // top: the lane's largest logit above M; returns what comes on top of logits above M.
    auto move = [&](int i, float top) {
      const bool none = most[i] == kNone;
      const float to = fmaxf(none ? -INFINITY : M[i] + (float)kOff, ceilf(max_of_row(top) + M[i]));
      const float Mn = to == -INFINITY ? 0.0f : to - (float)kOff;
      const float shift = M[i] - Mn;
      scale(i, none ? 0.0f : __builtin_amdgcn_exp2f(shift));
      M[i] = Mn;
      most[i] = to == -INFINITY ? kNone : (float)kOff + kSlack;
      return shift;
    };

    // ---- 16-bit tokens ----
    for (int u = piece; u < n_tail; u += step) {
      const bool win = u < n_win;
      const int t0 = (win ? u : u - n_win) * TAIL, count = win ? res : n_new;
      const size_t head = (size_t)b * Hkv + kvh;
      const uint16_t *kb, *vb;
      size_t stride;
      if (win) {
        kb = reinterpret_cast<const uint16_t*>(P.c.res_k) + head * R * D;
        vb = reinterpret_cast<const uint16_t*>(P.c.res_v) + head * R * D;
        stride = D;
      } else {
        kb = reinterpret_cast<const uint16_t*>(P.k_new) + ((size_t)b * P.T * Hkv + kvh) * D;
        vb = reinterpret_cast<const uint16_t*>(P.v_new) + ((size_t)b * P.T * Hkv + kvh) * D;
        stride = (size_t)Hkv * D;
      }
      // logits: tile j holds tokens t0 + 16 j .., row n of the tile = token n of it
      u32x4 ka[2][4];
      float norm[2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint16_t* row = kb + (size_t)min(t0 + 16 * j + n, count - 1) * stride + 32 * q4;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) ka[j][kk] = *reinterpret_cast<const u32x4*>(row + 8 * kk);
#pragma unroll
        for (int r = 0; r < 4; ++r) norm[j][r] = load_meta(P.c.res_norm, head * R + min(t0 + 16 * j + 4 * q4 + r, R - 1), MB);
      }
      // Values: rows of 64 channels in, a lane 8 channels of four tokens; through LDS, and columns of four tokens out.
      // (Loaded as columns, 64 times two bytes a lane, and with one limb 500 new tokens over 2 x 8100 4-bit took 225 us, 207
      // so; 2000 over 130 271 and 159.)
      u32x4 va[4];
      auto load_values = [&](int half) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          va[i] = *reinterpret_cast<const u32x4*>(vb + (size_t)min(t0 + 8 * i + lane / 8, count - 1) * stride + 64 * half +
                                                  8 * (lane % 8));
        __builtin_amdgcn_sched_barrier(0);
      };
      __builtin_amdgcn_sched_barrier(0);   // (all loads before the first use; left alone they go out one by one)
      float4v s[NR][2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        u32x4 (&a)[4] = ka[j];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          float4v acc = {0, 0, 0, 0};
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            if (win) {
              acc = mfma(__builtin_bit_cast(half8, a[kk]), lds.loop.qh[i][0][kk][lane], acc);
              acc = mfma(__builtin_bit_cast(half8, a[kk]), lds.loop.qh[i][1][kk][lane], acc);
            } else {
              const u32x4 r = lds.loop.q[i][kk][lane];
              if (bf16)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[kk]),
                                                              __builtin_bit_cast(bf16x8, r), acc, 0, 0, 0);
              else
                acc = mfma(__builtin_bit_cast(half8, a[kk]), __builtin_bit_cast(half8, r), acc);
            }
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int tok = t0 + 16 * j + 4 * q4 + r;
            s[i][j][r] = tok < count && (win || tok <= row_t[i]) ? acc[r] * (win ? norm[j][r] * q_unit[i] : P.scale_log2) : -INFINITY;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const float top = fmaxf(fmaxf(fmaxf(s[i][0][0], s[i][0][1]), fmaxf(s[i][0][2], s[i][0][3])),
                                fmaxf(fmaxf(s[i][1][0], s[i][1][1]), fmaxf(s[i][1][2], s[i][1][3]))) - M[i];
        if (__any(top > most[i])) move(i, top);
      }
      // Probabilities: two fp16 limbs beside fp16 values, two bf16 ones beside bf16 values, whose range is an fp32's: 2^-18
      // of each, where the outputs are rounded to 2^-9 of themselves (a third limb: 2000 new tokens over 130 183 -> 174 us
      // without it).
      half8 pr[NR][2];   // (16 bits of either type)
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        float p[8];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) p[4 * j + r] = __builtin_amdgcn_exp2f(s[i][j][r] - M[i]);
        if (bf16) {
          const bf16x8 one = (__bf16)(n == 4 ? 1.0f : 0.0f);
#pragma unroll
          for (int limb = 0; limb < 2; ++limb) {
            bf16x8 b;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              b[e] = (__bf16)p[e];
              p[e] -= (float)b[e];
            }
            x[i] = mfma(one, b, x[i]);
            pr[i][limb] = __builtin_bit_cast(half8, b);
          }
        } else {
          const half8 one = (_Float16)(n == 4 ? 1.0f : 0.0f);
          Limbs two;
#pragma unroll
          for (int e = 0; e < 8; e += 2) split2(p[e], p[e + 1], two, e);
          x[i] = mfma(one, two.hi, x[i]);
          x[i] = mfma(one, two.lo, x[i]);
          pr[i][0] = two.hi, pr[i][1] = two.lo;
        }
      }
      load_values(0);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        wave_lds_fence();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          half8 a;
          if (bf16) {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float lo = __builtin_amdgcn_fmed3f(__uint_as_float(va[i][e] << 16), -kBf16Most, kBf16Most);
              const float hi = __builtin_amdgcn_fmed3f(__uint_as_float(va[i][e] & 0xffff0000u), -kBf16Most, kBf16Most);
              w[e] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
            }
            a = __builtin_bit_cast(half8, w);
          } else {
            const half8 most = (_Float16)kHalfMax;
            a = __builtin_elementwise_min(__builtin_elementwise_max(__builtin_bit_cast(half8, va[i]), -most), most);
          }
          lds.loop.of_wave[wave].tail[8 * i + lane / 8][lane % 8] = a;
        }
        if (half == 0) load_values(1);
        wave_lds_fence();
        // channel 64 half + 16 ct + n of tokens t0 + 16 j + 4 q4 + r: columns of what was written as rows
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) {
          half8 a;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const auto at = (__attribute__((address_space(3))) short4v*)(reinterpret_cast<_Float16*>(
                                &lds.loop.of_wave[wave].tail[16 * j + 4 * q4 + n / 4][0]) + 16 * ct + 4 * (n % 4));
            const half4v four = __builtin_bit_cast(half4v, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at));
#pragma unroll
            for (int r = 0; r < 4; ++r) a[4 * j + r] = four[r];
          }
#pragma unroll
          for (int i = 0; i < NR; ++i) {
            float4v& acc = o[i][4 * half + ct];
            if (bf16) {
#pragma unroll
              for (int limb = 0; limb < 2; ++limb) acc = mfma(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, pr[i][limb]), acc);
            } else {
              acc = mfma(a, pr[i][0], acc);
              acc = mfma(a, pr[i][1], acc);
            }
          }
        }
      }
    }

    // ---- pages ----
    constexpr float kCodeUnit = 1.0f / (float)(1 << (24 - C::BPMIN));     // of a code in the sums
    wave_lds_fence();                                                     // (the last piece's values have been read)
    if (lane < 16) {
      meta.v_zero[0][64 + lane] = lane / 4 % 2 == 0 ? C::counterweight(0) : C::counterweight(1);
      meta.v_zero[1][64 + lane] = (half8)(_Float16)0.0f;
    }
    stage_keys();
    int x_page = stage_values(-100), x_sum = x_page;   // of the page to come, of the sums
    wave_lds_fence();
    // of the group that channels 32 w .. are in
    auto of_group = [&](int v, int w) { return __builtin_amdgcn_readlane(v, 16 * (w * P.g.ngv >> 2)); };
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) o[i][ct] *= kCodeUnit * exp2i(-of_group(x_sum, ct / 2));
    const int gb = (n == 4 ? 64 : min(n, P.g.ngv - 1) * 16) + q4;         // this lane's row of the extra tile
    for (; page < pages; page += step) {
      const int entry = entry_of(page + 2 * step);
      const float gone = pg0.held ? 0.0f : INFINITY;   // what is no page: its numbers are finite, its probabilities zeros
      if (__any(x_page != x_sum)) [[unlikely]] {   // the page's value steps are larger than any before
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float by = exp2i(max(of_group(x_sum, w) - of_group(x_page, w), -126));
#pragma unroll
          for (int i = 0; i < NR; ++i) o[i][2 * w] *= by, o[i][2 * w + 1] *= by;
        }
        // (rows 0 .. 3 of the extra tile: groups 0 .. 3)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * min(r, P.g.ngv - 1);
          const int by = __builtin_amdgcn_readlane(x_sum, row) - __builtin_amdgcn_readlane(x_page, row);
#pragma unroll
          for (int i = 0; i < NR; ++i) x[i][r] *= q4 == 0 ? exp2i(max(by, -126)) : 1.0f;
        }
        x_sum = x_page;
      }
      // Logits.  The queries' products with the steps are made for one k-step at a time, for SPAN quarters of the
      // page's tokens: for all k-steps at once they take registers that are not there.
      constexpr int SPAN = ONE ? AHEAD : 1;
      float4v s[NR][8];
      float4v start[NR];
      int q_lane = lane;
#pragma unroll
      for (int w0 = 0; w0 < 4; w0 += SPAN) {
        const int gk = ONE ? 0 : (w0 * P.g.ngk >> 2) * 16;
        if (!ONE || w0 == 0) {
          // what the zero terms add to every token of the group
#pragma unroll
          for (int i = 0; i < NR; ++i) start[i] = (float4v){0, 0, 0, 0};
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            const half8 zh = meta.k_zero[0][gk + 4 * q4 + kk], zl = meta.k_zero[1][gk + 4 * q4 + kk];
#pragma unroll
            for (int i = 0; i < NR; ++i) {
              const half8 qh = lds.loop.qc[i][0][kk][q_lane], ql = lds.loop.qc[i][1][kk][q_lane];
              start[i] = mfma(zh, qh, start[i]);
              start[i] = mfma(zh, ql, start[i]);
              start[i] = mfma(zl, qh, start[i]);
            }
          }
#pragma unroll
          for (int i = 0; i < NR; ++i) start[i] *= kCodeUnit;
        }
        asm("" : "+v"(q_lane));   // (read again: kept, the queries fill the registers)
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          half8 st[2];
          st[0] = meta.k_step[0][gk + 4 * q4 + kk];
          if (M32) st[1] = meta.k_step[M32 ? 1 : 0][gk + 4 * q4 + kk];
          Limbs qd[NR];
#pragma unroll
          for (int i = 0; i < NR; ++i) qd[i] = times<M32>(lds.loop.qc[i][0][kk][q_lane], lds.loop.qc[i][1][kk][q_lane], st);
#pragma unroll
          for (int t = 2 * w0; t < 2 * (w0 + SPAN); ++t) {
            const half8 a = C::operand(kc[t / 2] + t % 2 * BITS, kk);
#pragma unroll
            for (int i = 0; i < NR; ++i) s[i][t] = mfma(a, qd[i].hi, kk == 0 ? start[i] : s[i][t]);
#pragma unroll
            for (int i = 0; i < NR; ++i) s[i][t] = mfma(a, qd[i].lo, s[i][t]);
          }
        }
        if (AHEAD < 4 && w0 == 0 && SPAN == AHEAD) load_codes(pool_of(P.c.v_codes, code_shift, pg0), v_at, vc, AHEAD, 4);
        if (AHEAD < 4 && w0 == 1 && SPAN == 1) load_codes(pool_of(P.c.v_codes, code_shift, pg0), v_at, vc, AHEAD, 4);
      }
      if (!LATE) {
        load_codes(pool_of(P.c.k_codes, code_shift, pg1), k_at, kc, 0, AHEAD);
        fetch_meta(pg1);
      }
      // logits above M, less the bit position's exponent; what is no page has none
      float top[NR], unit[NR];
#pragma unroll
      for (int i = 0; i < NR; ++i) top[i] = -INFINITY, unit[i] = q_unit[i] * (float)(1 << (24 - C::BPMIN));
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float4v nm = *reinterpret_cast<const float4v*>(&meta.norm[(4 * r + q4) * 8 + 4 * half]);
#pragma unroll
          for (int i = 0; i < NR; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              s[i][4 * half + t][r] = fmaf(s[i][4 * half + t][r], nm[t] * unit[i], -(M[i] + ((float)C::above(r, 4 * half + t) + gone)));
              top[i] = fmaxf(top[i], s[i][4 * half + t][r]);
            }
        }
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        if (!__any(top[i] > most[i])) continue;
        float most_of = -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int t = 0; t < 8; ++t) most_of = fmaxf(most_of, s[i][t][r] + (float)C::above(r, t));
        const float shift = move(i, most_of);
#pragma unroll
        for (int t = 0; t < 8; ++t) s[i][t] += shift;
      }
      Limbs pr[NR][4];
#pragma unroll
      for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int t = 0; t < 8; t += 2)
            split2(__builtin_amdgcn_exp2f(s[i][t][r]), __builtin_amdgcn_exp2f(s[i][t + 1][r]), pr[i][r], t);

      // values
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const half8 zh = meta.v_zero[0][gb + 4 * kk], zl = meta.v_zero[1][gb + 4 * kk];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          x[i] = mfma(zh, pr[i][kk].hi, x[i]);
          x[i] = mfma(zh, pr[i][kk].lo, x[i]);
          x[i] = mfma(zl, pr[i][kk].hi, x[i]);
        }
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int gv = w * P.g.ngv >> 2;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          half8 st[2];
          st[0] = meta.v_step[0][gv * 16 + 4 * kk + q4];
          if (M32) st[1] = meta.v_step[M32 ? 1 : 0][gv * 16 + 4 * kk + q4];
          Limbs pd[NR];
#pragma unroll
          for (int i = 0; i < NR; ++i) pd[i] = times<M32>(pr[i][kk].hi, pr[i][kk].lo, st);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const half8 a = C::operand(vc[w] + j * BITS, kk);
#pragma unroll
            for (int i = 0; i < NR; ++i) o[i][2 * w + j] = mfma(a, pd[i].hi, o[i][2 * w + j]);
#pragma unroll
            for (int i = 0; i < NR; ++i) o[i][2 * w + j] = mfma(a, pd[i].lo, o[i][2 * w + j]);
          }
        }
        if (w == 1 && LATE) {
          load_codes(pool_of(P.c.k_codes, code_shift, pg1), k_at, kc, 0, AHEAD);
          fetch_meta(pg1);
        }
      }
      if (AHEAD < 4) load_codes(pool_of(P.c.k_codes, code_shift, pg1), k_at, kc, AHEAD, 4);
      load_codes(pool_of(P.c.v_codes, code_shift, pg1), v_at, vc, 0, AHEAD);
      wave_lds_fence();
      stage_keys();
      x_page = stage_values(x_sum);
      wave_lds_fence();
      pg0 = pg1;
      pg1 = page_of(page + 2 * step, entry);
    }
    // back to numbers: codes' unit, exponents, zero terms of each channel's value group
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      float zb[4];   // of channels 32 w .. 32 w + 31
#pragma unroll
      for (int gv = 0; gv < 4; ++gv) zb[gv] = __shfl(x[i][gv], n, 64);
      if (P.g.ngv == 2) zb[3] = zb[2] = zb[1];
      if (P.g.ngv < 4) zb[1] = zb[0];
      if (P.g.ngv == 1) zb[3] = zb[2] = zb[0];
#pragma unroll
      for (int ct = 0; ct < 8; ++ct)
        o[i][ct] = (o[i][ct] * (float)(1 << (24 - C::BPMIN)) + zb[ct / 2]) * exp2i(of_group(x_sum, ct / 2));
    }
    __syncthreads();
  }

  // ---- the four waves joined ----
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const float l = __shfl(x[i][0], 16 + n, 64);
    if (q4 == 0) {
      lds.join.m[wave][16 * i + n] = most[i] == kNone ? -INFINITY : M[i];
      lds.join.l[wave][16 * i + n] = l;
    }
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) *reinterpret_cast<float4v*>(&lds.join.o[wave][16 * i + n][16 * ct + 4 * q4]) = o[i][ct];
  }
  __syncthreads();
  const int c4 = (tid & 31) * 4;
  for (int row = tid >> 5; row < ROWS; row += 8) {
    if (row0 + row >= P.T * g) break;
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) mx = fmaxf(mx, lds.join.m[w][row]);
    float4v y = {0, 0, 0, 0};
    float l = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (lds.join.m[w][row] == -INFINITY) continue;
      const float f = __builtin_amdgcn_exp2f(lds.join.m[w][row] - mx);
      y += *reinterpret_cast<const float4v*>(&lds.join.o[w][row][c4]) * f;
      l = fmaf(lds.join.l[w][row], f, l);
    }
    const bool there = row < rows;
    const int t = P.by_group.of(row0 + row), h = kvh * g + (row0 + row - t * g);
    const size_t out_row = ((size_t)b * P.T + t) * Hq + h;
    if (!there) y = (float4v){0, 0, 0, 0};
    if (P.num_splits > 1) {
      float* rec = P.ws + (out_row * P.num_splits + split) * WS_STRIDE;
      *reinterpret_cast<float2v*>(rec + c4) = (float2v){y[0], y[1]};
      *reinterpret_cast<float2v*>(rec + c4 + 2) = (float2v){y[2], y[3]};
      if (c4 == 0) *reinterpret_cast<float2v*>(rec + D) = there ? (float2v){mx, l} : (float2v){-INFINITY, 0};
    } else {
      const float inv = l > 0.0f ? 1.0f / l : 0.0f;
      uint16_t v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[e] = bf16 ? __builtin_bit_cast(uint16_t, __float2bfloat16(y[e] * inv))
                    : __builtin_bit_cast(uint16_t, __float2half_rn(y[e] * inv));
      *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(P.out) + out_row * D + c4) =
          make_uint2(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16);
    }
  }
}

// A workgroup of NR tiles.  LAST: the second and last block of rows is 16 of them at most and takes one tile (35 rows,
// seven query heads and five tokens, over 131001 tokens: 50 us, 60 as twice two tiles; with G_k = 32 57 and 71).  Not
// with 4-bit codes, whose second body costs the first one more registers.
template <int BITS, bool M32, bool ONE, int NR, bool LAST>
__global__ __launch_bounds__(256, 2) void oscar_draft_kernel(DraftParams P) {
  __shared__ __align__(16) Lds<NR, M32> lds;
  const int row0 = (P.last_first ? gridDim.y - 1 - blockIdx.y : blockIdx.y) * NR * 16;
  if constexpr (LAST) {
    if (row0 > 0)
      attend<BITS, M32, ONE, 1>(P, reinterpret_cast<Lds<1, M32>&>(lds), row0);
    else
      attend<BITS, M32, ONE, NR>(P, lds, row0);
  } else {
    attend<BITS, M32, ONE, NR>(P, lds, row0);
  }
}

template <int BITS, bool M32, bool ONE> void launch(const DraftParams& P, int nr, dim3 grid, hipStream_t st) {
  const int64_t rows = (int64_t)P.T * P.group;
  if (nr == 1)
    hipLaunchKernelGGL((oscar_draft_kernel<BITS, M32, ONE, 1, false>), grid, dim3(256), 0, st, P);
  else if (BITS == 2 && rows > 32 && rows <= 48)
    hipLaunchKernelGGL((oscar_draft_kernel<BITS, M32, ONE, 2, BITS == 2>), grid, dim3(256), 0, st, P);
  else
    hipLaunchKernelGGL((oscar_draft_kernel<BITS, M32, ONE, 2, false>), grid, dim3(256), 0, st, P);
}
template <int BITS, bool M32> void launch(const DraftParams& P, int nr, dim3 grid, hipStream_t st) {
  if (P.g.ngk == 1)
    launch<BITS, M32, true>(P, nr, grid, st);
  else
    launch<BITS, M32, false>(P, nr, grid, st);
}

// Tiles of 16 query rows a wave holds: two read every page half as often (32 rows over 8 x 32K 100 us, 111 with one; 500
// new tokens of 32 heads over 2 x 8100 305 and 359, 4-bit 323 and 383), one has no idle half (16 rows 60 us, 89 with
// two; 4-bit 70 and 111).
int row_tiles(const oscar_config& cfg, int T) { return (int64_t)T * (cfg.n_q_heads / cfg.n_kv_heads) <= 16 ? 1 : 2; }
int64_t row_blocks(const oscar_config& cfg, int T) {
  const int rows = 16 * row_tiles(cfg, T);
  return ((int64_t)T * (cfg.n_q_heads / cfg.n_kv_heads) + rows - 1) / rows;
}

int check_draft_config(const oscar_config* cfg) {
  const int rc = oscar_validate_config(cfg);
  if (rc != OSCAR_OK) return rc;
  return cfg->io_dtype == OSCAR_F32 ? OSCAR_ERR_UNSUPPORTED : OSCAR_OK;
}

}  // namespace

// The split count whose estimate is the shortest.  A wave takes a piece (a page, or 32 tokens of the window or of the
// new ones) in 3 with one tile of rows and in 4 with two, 1.4 times that with 4-bit codes; workgroups that share a
// CU take 0.75 times as long each as one after the other; a workgroup's start costs 2 more.  Splitting costs the
// reduce pass: 3, 0.0004 a record, and past 64 splits 1.5 and 0.07 each (another kernel).  These are weights for the
// choice, in us to begin with; a call takes 1.7 times the estimate in the median (1.0 .. 3.5).  Over 186 calls of 1 .. 64
// sequences, 30 .. 131001 tokens and 1 .. 128 new ones the choice takes 0.9 % longer than the best count (14 at the
// most); weights nearer to the times (4.5 and 7 a piece) 1.3 % (24).
extern "C" int32_t oscar_draft_auto_splits(const oscar_config* cfg, int32_t batch, int32_t T, int32_t max_seq_len) {
  if (check_draft_config(cfg) != OSCAR_OK || batch <= 0 || T <= 0) return 1;
  const int64_t units = (int64_t)batch * cfg->n_kv_heads * row_blocks(*cfg, T), cus = oscar_compute_units();
  const int64_t len = max_seq_len > 0 ? max_seq_len : 0;
  const int64_t pieces = len / R + (len % R + TAIL - 1) / TAIL + ((int64_t)T + TAIL - 1) / TAIL;
  const float piece_us = (row_tiles(*cfg, T) == 1 ? 3.0f : 4.0f) * (cfg->bits == 4 ? 1.4f : 1.0f);
  const float record_us = 4e-4f * (float)batch * (float)T * (float)cfg->n_q_heads;
  float best = INFINITY;
  int32_t splits = 1;
  for (int32_t s = 1; s <= 512 && s <= (pieces + 3) / 4; s += s < 64 ? 1 : 8) {
    const int64_t share = (units * s + cus - 1) / cus;   // workgroups a CU
    const float us = (float)share * ((float)((pieces + 4 * s - 1) / (4 * s)) * piece_us * (share > 1 ? 0.75f : 1.0f) + 2.0f) +
                     (s > 1 ? 3.0f + record_us * (float)s : 0.0f) + (s > 64 ? 1.5f + 0.07f * (float)(s - 64) : 0.0f);
    if (us < best) best = us, splits = s;
    if (share > 8) break;   // no better from here on: more starts, and the same pages
  }
  return splits;
}

extern "C" size_t oscar_draft_workspace_bytes(const oscar_config* cfg, int32_t batch, int32_t T, int32_t num_splits) {
  if (!cfg || batch <= 0 || T <= 0 || num_splits <= 1 || cfg->n_q_heads <= 0) return 0;
  return (size_t)batch * T * cfg->n_q_heads * num_splits * WS_STRIDE * sizeof(float);
}

extern "C" int oscar_draft_attn(const void* q, const void* k_new, const void* v_new, int32_t T,
                                const int32_t* new_lens, const oscar_cache* cache, void* out,
                                float softmax_scale, int32_t max_seq_len_hint, int32_t num_splits,
                                void* workspace, size_t workspace_bytes, void* stream) {
  int rc = oscar_check_cache(cache);
  if (rc != OSCAR_OK) return rc;
  const oscar_config& cfg = cache->cfg;
  rc = check_draft_config(&cfg);
  if (rc != OSCAR_OK) return rc;
  if (T < 0 || max_seq_len_hint < 0 || num_splits < 0 || num_splits > 512 || cache->num_pages <= 0)
    return OSCAR_ERR_INVALID_ARG;
  if (T == 0) return OSCAR_OK;
  if (!q || !k_new || !v_new || !out) return OSCAR_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k_new) | reinterpret_cast<uintptr_t>(v_new) |
        reinterpret_cast<uintptr_t>(out)) & 15) != 0)
    return OSCAR_ERR_INVALID_ARG;
  if (num_splits == 0) num_splits = oscar_draft_auto_splits(&cfg, cache->batch, T, max_seq_len_hint);
  const int64_t blocks = row_blocks(cfg, T), units = (int64_t)cache->batch * cfg.n_kv_heads * num_splits;
  // (a launch takes 65535 blocks behind the first dimension and fewer than 2^32 threads along it)
  if (blocks > 65535 || units >= 1 << 24 || cache->batch > 65535 || (int64_t)T * cfg.n_q_heads >= 1 << 24)
    return OSCAR_ERR_INVALID_ARG;
  const size_t need = oscar_draft_workspace_bytes(&cfg, cache->batch, T, num_splits);
  if (need > 0 && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 7) != 0))
    return OSCAR_ERR_WORKSPACE;
  DraftParams P;
  P.q = q;
  P.k_new = k_new;
  P.v_new = v_new;
  P.out = out;
  P.ws = reinterpret_cast<float*>(workspace);
  P.new_lens = new_lens;
  P.c = *cache;
  P.g = make_geom(cfg.bits, cfg.k_group, cfg.v_group, cfg.meta_dtype);
  P.T = T;
  P.num_splits = num_splits;
  P.group = cfg.n_q_heads / cfg.n_kv_heads;
  // Where the new tokens outnumber the cached ones the last rows, which see the most of them, go first (2000 over 130:
  // 170 us, 197 the other way round); elsewhere that gains nothing, and ragged new_lens, whose empty blocks then come
  // first, lose (24 and 269 new tokens over 8100 and 5394, 4-bit: 186 us, 173 in the rows' order).
  // A hint of 0 is a length that is not known.
  P.last_first = max_seq_len_hint > 0 && T > max_seq_len_hint;
  P.by_splits = divisor(num_splits);
  P.by_step = divisor(4 * num_splits);
  P.by_kv_heads = divisor(cfg.n_kv_heads);
  P.by_group = divisor(P.group);
  P.scale_log2 = (softmax_scale > 0.0f ? softmax_scale : 0.08838834764831845f) * 1.4426950408889634f;
  // row blocks of one page range are a multiple of the XCDs' number apart wherever the ranges are
  const dim3 grid((unsigned)units, (unsigned)blocks);
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const int nr = row_tiles(cfg, T);
  const bool m32 = cfg.meta_dtype == OSCAR_F32;
  if (cfg.bits == 2) {
    if (m32) launch<2, true>(P, nr, grid, st); else launch<2, false>(P, nr, grid, st);
  } else {
    if (m32) launch<4, true>(P, nr, grid, st); else launch<4, false>(P, nr, grid, st);
  }
  if (num_splits > 1)
    oscar_launch_decode_reduce(P.ws, out, num_splits, cfg.io_dtype, T * cfg.n_q_heads, cache->batch, st);
  if (hipGetLastError() != hipSuccess) return OSCAR_ERR_HIP;
  return OSCAR_OK;
}
