// oscar_draft_attn: attention of several new tokens of every sequence over its packed cache and, causally,
// over each other.
//
//   logit[t][h][i] = scale n_i sum_j Q_j (Delta_k c_k - Delta_k z_k)_ij   cached token i, Q = H(q_th)/sqrt(128)
//                                                                        (float zero-points: Delta_k c_k + zero)
//   logit[t][h][j] = scale <q_th, k_j>                                   new token j <= t
//   out[t][h]      = softmax over both, times the values
//
// The T tokens' g query heads of a kv head are T g rows that read the same keys and values.  A workgroup
// takes 16 .. 64 of them (16 a matrix tile) through a share of the sequence, page by page:
//   wave w: S^T = K Q^T for tokens 32 w .. + 31   v_mfma_f32_16x16x32_f16, rows = tokens, columns = query rows
//   the rows' maxima through LDS, barrier; probabilities to LDS, barrier
//   wave w: O^T = V^T P^T for channels 32 w .. + 31, over all 128 tokens
// so that each code is loaded and unpacked once a workgroup, a wave's share of the keys lies in one group of
// tokens and that of the values in one group of channels, and the state of a row (16 registers a tile in all)
// leaves room for several workgroups a CU, which cover each other's barriers and loads.
//
// Row n of a token tile is token 4 (n % 4) + n / 4 of it: a lane's four results of tile T are then its tokens
// 16 T + 4 r + lane / 16, exactly those whose value codes the lane's chunk of the page holds for k-step r, and a
// lane reads the probabilities it multiplies with as 16 consecutive bytes.
//
// Codes become fp16 operands with a mask (a code parked in the mantissa of a subnormal: c 2^(s - 24)); the
// steps go to the other operand, Q Delta_k and P Delta_v, and 2^-s with them.  Codes count from their middle:
// the term that takes it off again is a product of the same rounded operands with a constant, what is left of
// the zero-points is of the size of a group's mean, and both are products on the matrix cores too: for the keys
// what a tile's sums start from, for the values one extra tile, whose other rows are the rows' sums.  Seen from
// code 0 the same roundings moved the logits three times as far.  Roundings: Q, Q Delta, P, P Delta and the
// mean terms to fp16, half a step (2^-11) each.  The probabilities are scaled by 2^9 .. 2^15 (less where a value
// step of 2 or more would carry P Delta past the fp16 range): a token counts down to 2^-33 of the largest.  Sums,
// maxima and outputs are fp32.
#include "oscar_decode_common.h"

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kHalfMax = 65504.0f;
constexpr int kQShift = 2;           // the queries carry 2^2

struct DraftParams {
  const void *q, *k_new, *v_new;
  void* out;
  float* ws;
  const int32_t* new_lens;
  oscar_cache c;
  PageGeom g;
  int T, num_splits;
  float scale_log2;
};

template <int BITS> struct Codes {
  static constexpr int BPMIN = BITS == 2 ? 4 : 2, BPMAX = BITS == 2 ? 8 : 6;
  static constexpr float MID = 0.5f * (float)((1 << BITS) - 1);
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
  // 2^(above - (BPMAX - BPMIN)), the other operand's counterweight for what is no code (kk counts modulo 2)
  __device__ static __forceinline__ half8 counterweight(int kk) {
    half8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (_Float16)(1.0f / (float)(1 << (BPMAX - BPMIN - above(kk, e))));
    return r;
  }
};

// A page's metadata as the waves read it: steps and mean terms (with their counterweights) as fp16 in operand
// order, norms as fp32 with the codes' unit taken out.
struct Staged {
  half8 k_step[64], k_base[64];   // [group][quarter][k-step]
  half8 v_step[64], v_base[80];   // [group][k-step][quarter]; behind the four groups the counterweights alone
  float norm[R];                  // position (token % 16) * 8 + token / 16
  int off;                        // exponent the probabilities can carry
};
// A row's probabilities are taken against a reference that follows its maximum only when that has passed it by
// 2^kSlack: over long sequences the maximum creeps up in many small steps, and each costs the workgroup a
// barrier and a rescaling.
constexpr float kSlack = 6.0f, kNone = -3e38f;
constexpr int kOff = 9;          // exponent of a probability at its reference: kOff + kSlack stay inside fp16
// What a lane holds of the metadata of a page to come: 8 steps and 8 zeros (wave 0 of the keys, wave 1 of the
// values) or 8 norms (the others).  All waves make the same loads, so that how many are in flight is known
// wherever one is waited for.
template <bool M32> struct Fetched {
  u32x4 a[M32 ? 2 : 1], b[M32 ? 2 : 1];
  __device__ __forceinline__ void load(const uint8_t* src, const uint8_t* zsrc, uint32_t at) {
#pragma unroll
    for (int i = 0; i < (M32 ? 2 : 1); ++i) {
      a[i] = *reinterpret_cast<const u32x4*>(src + at + 16 * i);
      b[i] = *reinterpret_cast<const u32x4*>(zsrc + at + 16 * i);
    }
  }
  __device__ __forceinline__ static float number(const u32x4* x, int e) {
    if (M32) return __uint_as_float(x[e / 4][e % 4]);
    return (float)__builtin_bit_cast(half8, x[0])[e];
  }
  // step and mean term: x = step (c - mid) + base
  __device__ __forceinline__ void step_and_base(bool zp_min, float mid, half8& step, half8& base) const {
    if (M32) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float s = number(a, e), z = number(b, e);
        step[e] = (_Float16)fminf(s, kHalfMax);
        base[e] = (_Float16)__builtin_amdgcn_fmed3f(zp_min ? fmaf(s, mid, z) : (mid - z) * s, -kHalfMax, kHalfMax);
      }
    } else {
      step = __builtin_bit_cast(half8, a[0]);
      const half8 z = __builtin_bit_cast(half8, b[0]), most = (_Float16)kHalfMax;
      const uint32_t two = __builtin_bit_cast(uint32_t, (half2v)(_Float16)mid);
      u32x4 w = {two, two, two, two};
      asm("" : "+v"(w));   // (as a constant it is taken apart into single halves)
      const half8 m = __builtin_bit_cast(half8, w);
      base = zp_min ? __builtin_elementwise_fma(step, m, z) : (m - z) * step;
      base = __builtin_elementwise_min(__builtin_elementwise_max(base, -most), most);
    }
  }
};

__device__ __forceinline__ float4v mfma(half8 a, half8 b, float4v c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v){a, b}, half2v));
}
__device__ __forceinline__ float max_of_row(float v) {   // over the four lanes that hold a query row
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// Workgroups a CU that a variant's registers are held to.
__host__ __device__ constexpr int wgs_per_cu(int nr) { return nr == 1 ? 4 : nr == 2 ? 3 : 2; }

template <int BITS, bool M32, int NR>
__global__ __launch_bounds__(256, wgs_per_cu(NR)) void oscar_draft_kernel(DraftParams P) {
  using C = Codes<BITS>;
  constexpr int ROWS = NR * 16;
  constexpr int UNITS = C::BPMAX - C::BPMIN;         // log2 of what the counterweights leave in the extra tile
  __shared__ __align__(16) half8 s_qh[NR][4][64], s_qc[NR][4][64];   // queries as operands: natural order, codes' order
  __shared__ __align__(16) uint32_t s_p[2][NR][4][64][4];            // probabilities as operands
  __shared__ __align__(16) int s_flag[2][4];
  __shared__ __align__(16) float s_max[ROWS][4];
  __shared__ __align__(16) Staged s_meta[3];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, q4 = lane >> 4;
  const int Hkv = P.c.cfg.n_kv_heads, Hq = P.c.cfg.n_q_heads, g = Hq / Hkv;
  const int split = blockIdx.x % P.num_splits, unit = blockIdx.x / P.num_splits;
  const int kvh = unit % Hkv, b = unit / Hkv;
  const int row0 = blockIdx.y * ROWS;

  const int n_new = P.new_lens ? min(max(P.new_lens[b], 0), P.T) : P.T;
  const int seq_len = max(P.c.seq_lens[b], 0);
  const int res = min(max(P.c.res_lens[b], 0), min(R, seq_len));
  const int pages = min((seq_len - res) / R, P.c.max_pages_per_seq);
  const int rows = min(max(n_new * g - row0, 0), ROWS);         // of this block that are there
  const bool zp_min = P.c.cfg.zp_mode == OSCAR_ZP_MIN;
  const bool bf16 = P.c.cfg.io_dtype == OSCAR_BF16;
  const int row_of_tile = 4 * (n % 4) + n / 4;                  // token of a tile that this lane's row is

  float4v o[NR][2];   // channels 32 wave + 16 j + 4 q4 + r of row n, in units of the codes once pages have begun
  float4v x[NR];      // [0]: zero terms of the wave's value group, [1]: the row's sum
  float ref[NR];      // what the row's probabilities are taken against, log2 units
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    o[i][0] = o[i][1] = x[i] = (float4v){0, 0, 0, 0};
    ref[i] = kNone;
  }
  int off = kOff;

  if (rows > 0) {
    // what the pages are: tail units (window, then new tokens, 128 each) and packed pages, dealt to the splits
    const int last_t = (row0 + rows - 1) / g;                            // last new token any row here sees
    const int n_win = res > 0 ? 1 : 0;
    const int n_tail = n_win + (min(n_new, last_t + 1) + R - 1) / R;
    const int step = P.num_splits;
    int page = split < n_tail ? split + (n_tail - split + step - 1) / step * step - n_tail : split - n_tail;
    // (read as constant memory, by the scalar unit: a vector load's wait would be one for every load ahead)
    const auto table = reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(
        reinterpret_cast<uintptr_t>(P.c.block_table + (size_t)b * P.c.max_pages_per_seq));
    // Physical page of page p; what is none is marked (its metadata is staged as zeros and its tokens are left
    // out), and loads past the end take a page again: every iteration then makes the same loads.
    struct Page {
      int phys;
      bool held;
    };
    auto entry_of = [&](int p) { return table[min(max(p, 0), max(pages - 1, 0))]; };
    auto page_of = [&](int p, int phys) {
      const bool ok = phys >= 0 && phys < P.c.num_pages;
      return Page{ok ? phys : 0, ok && p < pages};
    };

    // ---- loads ahead ----
    uint32_t kc[2 * BITS], vc[2 * BITS];
    const size_t k_stride = (size_t)Hkv * P.g.k_codes_bytes, v_stride = (size_t)Hkv * P.g.v_codes_bytes;
    const uint8_t* k_pool = reinterpret_cast<const uint8_t*>(P.c.k_codes) + (size_t)kvh * P.g.k_codes_bytes;
    const uint8_t* v_pool = reinterpret_cast<const uint8_t*>(P.c.v_codes) + (size_t)kvh * P.g.v_codes_bytes;
    const uint32_t k_at = chunk_offset(BITS, 2 * wave, row_of_tile, q4), v_at = chunk_offset(BITS, 2 * wave, n, q4);
    auto load_codes = [&](const uint8_t* page, uint32_t at, uint32_t* w) {
#pragma unroll
      for (int j = 0; j < BITS / 2; ++j) *reinterpret_cast<u32x4*>(w + 4 * j) = *reinterpret_cast<const u32x4*>(page + at + 16 * j);
    };
    constexpr int MB = M32 ? 4 : 2;
    const int m_bytes = wave == 0 ? P.g.k_meta_bytes : wave == 1 ? P.g.v_meta_bytes : P.g.k_norms_bytes;
    const int m_groups = wave == 0 ? P.g.ngk : wave == 1 ? P.g.ngv : 1;
    const uint8_t* m_pool = reinterpret_cast<const uint8_t*>(wave == 0 ? P.c.k_meta : wave == 1 ? P.c.v_meta : P.c.k_norms) +
                            (size_t)kvh * m_bytes;
    const size_t m_stride = (size_t)Hkv * m_bytes;
    const uint32_t m_zero = wave < 2 ? (uint32_t)m_groups * 128 * MB : 0, m_at = (uint32_t)min(lane, 16 * m_groups - 1) * 8 * MB;
    Fetched<M32> f;
    auto fetch_meta = [&](const Page& pg) {
      const uint8_t* src = m_pool + pg.phys * m_stride;
      f.load(src, src + m_zero, m_at);
    };
    auto stage_meta = [&](Staged& s, bool held) {
      if (wave >= 2) {
        if (wave == 2 && lane < 16) {
          constexpr float unit_of_codes = (float)(1 << (24 - C::BPMIN - kQShift));
#pragma unroll
          for (int e = 0; e < 8; ++e) s.norm[8 * lane + e] = held ? f.number(f.a, e) * unit_of_codes : 0.0f;
        }
        return;
      }
      half8 st, base;
      f.step_and_base(zp_min, C::MID, st, base);
      const int kk = wave == 0 ? lane : lane / 4;
      base *= kk % 2 == 0 ? C::counterweight(0) : C::counterweight(1);
      if (!held) st = base = (half8)(_Float16)0.0f;
      if (wave == 0) {
        s.k_step[lane] = st;
        s.k_base[lane] = base;
        return;
      }
      s.v_step[lane] = st;
      s.v_base[lane] = base;
      // the exponent of the largest step (fp16 bits; steps are not negative), bit by bit over the wave
      uint32_t big = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t two = __builtin_bit_cast(u32x4, st)[e];
        big = max(big, max(two & 0xffffu, two >> 16));
      }
      uint64_t among = ~0ull;
      int exponent = 0;
#pragma unroll
      for (int bit = 14; bit >= 10; --bit) {
        const uint64_t have = __ballot(big >> bit & 1) & among;
        if (have) among = have, exponent |= 1 << (bit - 10);
      }
      if (lane == 0) s.off = kOff - max(exponent - 14, 0);
    };

    // page, page + 1 step, page + 2 steps: the codes of the first two and the metadata of all are on their way
    Page pg0 = page_of(page, entry_of(page)), pg1 = page_of(page + step, entry_of(page + step)),
         pg2 = page_of(page + 2 * step, entry_of(page + 2 * step));
    fetch_meta(pg0);
    load_codes(k_pool + pg0.phys * k_stride, k_at, kc);
    load_codes(v_pool + pg0.phys * v_stride, v_at, vc);

    // ---- queries: lane's row, channels 32 q4 .. + 31; wave i rotates tile i ----
    const uint16_t* q_row[NR];
    int row_t[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int row = row0 + 16 * i + n;
      row_t[i] = row / g;
      const bool there = row < n_new * g;
      q_row[i] = reinterpret_cast<const uint16_t*>(P.q) +
                 (((size_t)b * P.T + (there ? row_t[i] : 0)) * Hq + (size_t)kvh * g + (there ? row % g : 0)) * D + 32 * q4;
      if (wave != i) continue;
      float y[32];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(q_row[i] + 8 * u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint16_t v = (uint16_t)(w[e / 2] >> (16 * (e % 2)));
          const float t = bf16 ? __uint_as_float((uint32_t)v << 16) : __half2float(__ushort_as_half(v));
          y[8 * u + e] = there ? t : 0.0f;
        }
      }
      float mul = P.scale_log2 * (float)(1 << kQShift);
      if (P.c.cfg.rotation == OSCAR_ROTATION_ON) {
#pragma unroll
        for (int h = 1; h < 32; h <<= 1) {
#pragma unroll
          for (int u = 0; u < 32; ++u) {
            if ((u & h) == 0) {
              const float a = y[u], c = y[u | h];
              y[u] = a + c;
              y[u | h] = a - c;
            }
          }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const float sg = (q4 >> s) & 1 ? -1.0f : 1.0f;
#pragma unroll
          for (int u = 0; u < 32; ++u) {
            // (each call leaves the two lanes' numbers side by side in both)
            const uint32_t v = __float_as_uint(y[u]);
            const auto two = s == 0 ? __builtin_amdgcn_permlane16_swap(v, v, false, false)
                                    : __builtin_amdgcn_permlane32_swap(v, v, false, false);
            y[u] = fmaf(__uint_as_float(two[1]), sg, __uint_as_float(two[0]));
          }
        }
        mul *= 0.08838834764831845f;
      }
      half8 qh[4];
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int e = 0; e < 8; ++e) qh[kk][e] = (_Float16)(y[8 * kk + e] * mul);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        half8 qc;   // in the codes' order, with the counterweights of their bit positions
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int u = slot_index(BITS, kk, e);
          qc[e] = qh[u / 8][u % 8] * (_Float16)(1.0f / (float)(1 << C::above(kk, e)));
        }
        s_qh[i][kk][lane] = qh[kk];
        s_qc[i][kk][lane] = qc;
      }
    }
    if (wave == 3 && lane < 16) {
#pragma unroll
      for (int i = 0; i < 3; ++i) s_meta[i].v_base[64 + lane] = lane / 4 % 2 == 0 ? C::counterweight(0) : C::counterweight(1);
    }
    stage_meta(s_meta[0], pg0.held);
    fetch_meta(pg1);
    stage_meta(s_meta[1], pg1.held);
    fetch_meta(pg2);
    __syncthreads();

    // Probabilities to LDS, as operands; s[i][j][r]: logit (log2 units) of the wave's token 16 (2 wave + j) + 4 r + q4.
    // even, odd: weights' exponents of the k-steps; gone: infinite for what is no page (its numbers are finite),
    // whose probabilities are zeros.  They are written against the references as they stand; if a
    // wave finds a row past its reference, all join the rows' maxima, rescale and write them again.  What was
    // written two calls ago is free: between lies a barrier that everyone reaches behind its reads.
    int turn = 0;
    auto softmax = [&](const float4v (&s)[NR][2], int most_off, float even, float odd, float gone) {
      auto write = [&] {
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          const float M = ref[i] - (float)off;
          const float Mk[2] = {M + (even + gone), M + (odd + gone)};
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s_p[turn][i][r][lane][wave] = pack2(__builtin_amdgcn_exp2f(s[i][0][r] - Mk[r % 2]),
                                                __builtin_amdgcn_exp2f(s[i][1][r] - Mk[r % 2]));
        }
      };
      turn ^= 1;
      float mx[NR];
      bool past = most_off < off;
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        mx[i] = fmaxf(fmaxf(fmaxf(s[i][0][0], s[i][0][1]), fmaxf(s[i][0][2], s[i][0][3])),
                      fmaxf(fmaxf(s[i][1][0], s[i][1][1]), fmaxf(s[i][1][2], s[i][1][3])));
        past |= mx[i] > ref[i] + (kSlack + gone);
      }
      write();
      const int flag = __any(past);
      if (lane == 0) s_flag[turn][wave] = flag;
      __syncthreads();
      const u32x4 flags = *reinterpret_cast<const u32x4*>(s_flag[turn]);
      if (__builtin_amdgcn_readfirstlane(flags[0] | flags[1] | flags[2] | flags[3]) == 0) return;
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        mx[i] = max_of_row(mx[i]);
        if (q4 == 0) s_max[16 * i + n][wave] = mx[i];
      }
      __syncthreads();
      const int now = min(off, most_off);
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const float4v mw = *reinterpret_cast<const float4v*>(s_max[16 * i + n]);
        const float to = fmaxf(ref[i], fmaxf(fmaxf(mw[0], mw[1]), fmaxf(mw[2], mw[3])));
        const float alpha = __builtin_amdgcn_exp2f(ref[i] - to + (float)(now - off));
        o[i][0] *= alpha;
        o[i][1] *= alpha;
        x[i] *= alpha;
        ref[i] = to;
      }
      off = now;
      write();
      __syncthreads();
    };

    // ---- 16-bit tokens ----
    for (int u = split; u < n_tail; u += step) {
      const bool win = u < n_win;
      const int t0 = win ? 0 : (u - n_win) * R, count = win ? res : n_new;
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
      float4v s[NR][2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int tile0 = t0 + 16 * (2 * wave + j);
        if (tile0 < count) {
          const int t = min(tile0 + row_of_tile, count - 1);
          u32x4 a[4];
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) a[kk] = *reinterpret_cast<const u32x4*>(kb + (size_t)t * stride + 32 * q4 + 8 * kk);
#pragma unroll
          for (int i = 0; i < NR; ++i) {
            float4v acc = {0, 0, 0, 0};
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
              if (win) {
                acc = mfma(__builtin_bit_cast(half8, a[kk]), s_qh[i][kk][lane], acc);
              } else {
                const u32x4 r = *reinterpret_cast<const u32x4*>(q_row[i] + 8 * kk);
                if (bf16)
                  acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[kk]),
                                                                __builtin_bit_cast(bf16x8, r), acc, 0, 0, 0);
                else
                  acc = mfma(__builtin_bit_cast(half8, a[kk]), __builtin_bit_cast(half8, r), acc);
              }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int tok = tile0 + 4 * r + q4;
              const float fac = win ? load_meta(P.c.res_norm, head * R + min(tok, R - 1), M32 ? 4 : 2) * (1.0f / (1 << kQShift))
                                    : P.scale_log2;
              s[i][j][r] = tok < count && (win || tok <= row_t[i]) ? acc[r] * fac : -INFINITY;
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < NR; ++i) s[i][j] = (float4v){-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        }
      }
      softmax(s, off, 0.0f, 0.0f, 0.0f);
      // values: channel 32 wave + 16 j + n of tokens t0 + 16 e + 4 kk + q4
      const half8 one = (_Float16)(n % 4 == 1 ? 1.0f / (1 << UNITS) : 0.0f);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        half8 a[2];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int t = t0 + 16 * e + 4 * kk + q4;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float y = 0.0f;
            if (t0 + 16 * e < count) {
              const uint16_t v = vb[(size_t)min(t, count - 1) * stride + 32 * wave + 16 * j + n];
              y = bf16 ? __uint_as_float((uint32_t)v << 16) : __half2float(__ushort_as_half(v));
              y = t < count ? __builtin_amdgcn_fmed3f(y, -kHalfMax, kHalfMax) : 0.0f;
            }
            a[j][e] = (_Float16)y;
          }
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          const half8 p = *reinterpret_cast<const half8*>(s_p[turn][i][kk][lane]);
          o[i][0] = mfma(a[0], p, o[i][0]);
          o[i][1] = mfma(a[1], p, o[i][1]);
          x[i] = mfma(one, p, x[i]);
        }
      }
    }

    // ---- pages ----
    constexpr float kCodeUnit = 1.0f / (float)(1 << (24 - C::BPMIN));     // of a code in the sums
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      o[i][0] *= kCodeUnit;
      o[i][1] *= kCodeUnit;
    }
    // the wave's groups in the staged metadata, its probabilities' weights, constants of the middle
    const int gk = wave * 32 / P.g.k_group * 16, gv = wave * 32 / P.g.v_group * 16;
    const int gb = n % 4 == 1 ? 64 : gv;     // the extra tile's second row: the rows' sums
    const float even = (float)(BITS == 2 ? 2 * (wave % 2) : 4 * (wave % 2));
    const float odd = (float)(BITS == 2 ? (wave == 0 || wave == 3 ? 4 : 2 * (wave - 1)) : 4 * (wave % 2));
    for (int buf = 0; page < pages; page += step) {
      const Staged& meta = s_meta[buf];
      const int entry = entry_of(page + 3 * step);
      // logits
      float4v s[NR][2], start[NR];
      half8 qd[NR][4];
#pragma unroll
      for (int i = 0; i < NR; ++i) start[i] = (float4v){0, 0, 0, 0};
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const half8 st = meta.k_step[gk + 4 * q4 + kk], base = meta.k_base[gk + 4 * q4 + kk];
        const half8 mid = C::counterweight(kk) * (_Float16)-C::MID;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          const half8 qc = s_qc[i][kk][lane];
          qd[i][kk] = qc * st;
          start[i] = mfma(base, qc, start[i]);
          start[i] = mfma(mid, qd[i][kk], start[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < NR; ++i) s[i][0] = s[i][1] = start[i] * (1.0f / (float)(1 << (24 - C::BPMAX)));
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          const half8 a = C::operand(kc + j * BITS, kk);
#pragma unroll
          for (int i = 0; i < NR; ++i) s[i][j] = mfma(a, qd[i][kk], s[i][j]);
        }
      load_codes(k_pool + pg1.phys * k_stride, k_at, kc);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float2v nm = *reinterpret_cast<const float2v*>(&meta.norm[(4 * r + q4) * 8 + 2 * wave]);
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          s[i][0][r] *= nm[0];
          s[i][1][r] *= nm[1];
        }
      }
      softmax(s, __builtin_amdgcn_readfirstlane(meta.off), even, odd, pg0.held ? 0.0f : INFINITY);
      // values
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const half8 st = meta.v_step[gv + 4 * kk + q4], base = meta.v_base[gb + 4 * kk + q4];
        const half8 mid = C::counterweight(kk) * (_Float16)(n % 4 == 0 ? -C::MID : 0.0f);
        const half8 a0 = C::operand(vc, kk), a1 = C::operand(vc + BITS, kk);
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          const half8 p = *reinterpret_cast<const half8*>(s_p[turn][i][kk][lane]);
          const half8 pd = p * st;
          x[i] = mfma(base, p, x[i]);
          x[i] = mfma(mid, pd, x[i]);
          o[i][0] = mfma(a0, pd, o[i][0]);
          o[i][1] = mfma(a1, pd, o[i][1]);
        }
      }
      load_codes(v_pool + pg1.phys * v_stride, v_at, vc);
      // every wave has left the page before this one: its buffer takes the page after next
      const int into = buf == 0 ? 2 : buf - 1;
      stage_meta(s_meta[into], pg2.held);
      pg0 = pg1;
      pg1 = pg2;
      pg2 = page_of(page + 3 * step, entry);
      fetch_meta(pg2);
      buf = buf == 2 ? 0 : buf + 1;
    }
  }

  // ---- back to numbers, and out ----
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const int row = row0 + 16 * i + n;
    if (row >= P.T * g) continue;
    const bool there = 16 * i + n < rows;
    const float zero = x[i][0] * (float)(1 << UNITS), l = x[i][1] * (float)(1 << UNITS);
    const size_t out_row = ((size_t)b * P.T + row / g) * Hq + kvh * g + row % g;
    const float inv = there && l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int c = 32 * wave + 16 * j + 4 * q4;
      float4v y = o[i][j] * (float)(1 << (24 - C::BPMIN)) + zero;
      if (!there) y = (float4v){0, 0, 0, 0};
      if (P.num_splits > 1) {
        float* rec = P.ws + (out_row * P.num_splits + split) * WS_STRIDE + c;
        *reinterpret_cast<float2v*>(rec) = (float2v){y[0], y[1]};
        *reinterpret_cast<float2v*>(rec + 2) = (float2v){y[2], y[3]};
      } else {
        uint16_t v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = bf16 ? __builtin_bit_cast(uint16_t, __float2bfloat16(y[e] * inv))
                      : __builtin_bit_cast(uint16_t, __float2half_rn(y[e] * inv));
        *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(P.out) + out_row * D + c) =
            make_uint2(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16);
      }
    }
    if (P.num_splits > 1 && wave == 0 && q4 == 0)
      *reinterpret_cast<float2v*>(P.ws + (out_row * P.num_splits + split) * WS_STRIDE + D) =
          there && ref[i] > kNone ? (float2v){ref[i] - (float)off, l} : (float2v){-INFINITY, 0};
  }
}

template <int BITS, bool M32> void launch(const DraftParams& P, int nr, dim3 grid, hipStream_t st) {
  switch (nr) {
    case 1: hipLaunchKernelGGL((oscar_draft_kernel<BITS, M32, 1>), grid, dim3(256), 0, st, P); break;
    case 2: hipLaunchKernelGGL((oscar_draft_kernel<BITS, M32, 2>), grid, dim3(256), 0, st, P); break;
    case 3: hipLaunchKernelGGL((oscar_draft_kernel<BITS, M32, 3>), grid, dim3(256), 0, st, P); break;
    default: hipLaunchKernelGGL((oscar_draft_kernel<BITS, M32, 4>), grid, dim3(256), 0, st, P); break;
  }
}

// tiles of 16 query rows a workgroup takes
int row_tiles(const oscar_config& cfg, int T) {
  const int64_t tiles = ((int64_t)T * (cfg.n_q_heads / cfg.n_kv_heads) + 15) / 16;
  return tiles < 4 ? (int)tiles : 4;
}
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

extern "C" int32_t oscar_draft_auto_splits(const oscar_config* cfg, int32_t batch, int32_t T, int32_t max_seq_len) {
  if (check_draft_config(cfg) != OSCAR_OK || batch <= 0 || T <= 0) return 1;
  const int64_t units = (int64_t)batch * cfg->n_kv_heads * row_blocks(*cfg, T);
  const int64_t pages = max_seq_len > 0 ? ((int64_t)max_seq_len + R - 1) / R : 1;
  int64_t splits = wgs_per_cu(row_tiles(*cfg, T)) * (int64_t)oscar_compute_units() / units;
  if (splits > pages) splits = pages;
  if (splits > 512) splits = 512;
  return splits < 1 ? 1 : (int32_t)splits;
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
  if (blocks > 65535 || units > 0x7fffffff || cache->batch > 65535 || (int64_t)T * cfg.n_q_heads > 0x7fffffff)
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
