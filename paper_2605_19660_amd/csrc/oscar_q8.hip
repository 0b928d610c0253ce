// The paged 8-bit cache: oscar_q8_append, oscar_q8_read, sizes and checks.
//
//   a = max |x| over the block's tokens and channels (of one kv head, keys and values apart)
//   scale = 2^e, e = ceil(log2(a / 448)): with a = m 2^f, 1/2 <= m < 1, that is f - 9, or f - 8 where m > 7/8
//   code = e4m3(x / scale), to nearest, ties to even
// A power of two loses nothing against a / 448 with floating-point codes (three bits of mantissa at any
// scale; numbers 2^15 below the largest fall under the last step), the quotient is exact, so that a code does not
// depend on how it is worked out, and a code times its scale is exact in bf16.
//
// Append: a workgroup takes one block of one kv head, keys or values: reads it once (a new token's 256 bytes
// by 16 lanes, the tokens that were there from the window), finds the largest, converts in registers.  Four value
// tokens lie in four rows of 16 lanes of a wave and change places by half and quarter swaps of registers, because
// pages hold values channel by channel.  Bound by memory for prompts (4 x 8192 tokens of 8 kv heads: 37 .. 40 us, 5.0 .. 5.4
// TB/s read and written, a copy's own 5.1), by latency for single tokens (3 us).
//
// Read: a wave takes a step (32 tokens) of a kv head: codes in whole kilobytes, rows put together in LDS, 16 bytes
// a lane out.  Bound by writing rows: 4 x 16K tokens of fp16 as fp32 take 106 us, 5.1 TB/s read and written, a copy's own
// rate (85 where the last-level cache holds the codes); 4 x 8192 in bf16, just appended, 32 us, 2048 12.
#include "oscar_q8.h"

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t s16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

template <typename E> __device__ __forceinline__ float widen(uint32_t bits16);
template <> __device__ __forceinline__ float widen<__hip_bfloat16>(uint32_t b) { return bf16_bits_to_f32(b); }
template <> __device__ __forceinline__ float widen<__half>(uint32_t b) {
  return __half2float(__builtin_bit_cast(__half, (uint16_t)b));
}
template <typename E> __device__ __forceinline__ uint32_t narrow(float x) {
  return __builtin_bit_cast(uint16_t, from_f32<E>(x));
}

// What the cache takes at most, as a number's bits without its sign (an infinity and a NaN have more).
template <typename E> constexpr uint16_t MOST_BITS = __is_same(E, __half) ? 0x7bff : (127 + 60) << 7;
__device__ __forceinline__ u16x2 most_bits(u16x2 most, u32x4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu));
  return most;
}
// What counts for the numbers of a piece: NaN as 0, large ones as the largest.
template <typename E> __device__ __forceinline__ u32x4 counted(u32x4 v) {
  constexpr uint32_t nan = __is_same(E, __half) ? 0x7c00 : 0x7f80;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t out = 0;
#pragma unroll
    for (int s = 0; s < 32; s += 16) {
      const uint32_t bits = v[i] >> s & 0x7fff, sign = v[i] >> s & 0x8000;
      out |= (bits > nan ? 0 : sign | min(bits, (uint32_t)MOST_BITS<E>)) << s;
    }
    v[i] = out;
  }
  return v;
}
// Two numbers divided by a power of two, to the nearest e4m3 numbers.
template <typename E> __device__ __forceinline__ uint32_t two_codes(uint32_t old, uint32_t two, float scale, bool upper);
template <> __device__ __forceinline__ uint32_t two_codes<__hip_bfloat16>(uint32_t old, uint32_t two, float scale, bool upper) {
  const bf16x2 x = __builtin_bit_cast(bf16x2, two);
  const s16x2 o = __builtin_bit_cast(s16x2, old);
  return __builtin_bit_cast(uint32_t, upper ? __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, x, scale, true)
                                            : __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, x, scale, false));
}
template <> __device__ __forceinline__ uint32_t two_codes<__half>(uint32_t old, uint32_t two, float scale, bool upper) {
  const f16x2 x = __builtin_bit_cast(f16x2, two);
  const s16x2 o = __builtin_bit_cast(s16x2, old);
  return __builtin_bit_cast(uint32_t, upper ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(o, x, scale, true)
                                            : __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(o, x, scale, false));
}
template <typename E> __device__ __forceinline__ u32x4 narrow8(const float* x) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = narrow<E>(x[2 * i]) | narrow<E>(x[2 * i + 1]) << 16;
  return v;
}

struct AppendParams {
  Q8Cache c;
  Q8Rows r;
  const uint16_t *k, *v;
  int64_t k_stride, v_stride;
  int blocks;   // of a sequence, at most
};

// Lane (row i of 16 lanes, n) holds 8 channels of token 4 * q4 + i (two dwords); afterwards it holds tokens
// 4 * q4 + 0 .. 3 of channels 2 i and 2 i + 1 of the 8 (a dword each).
__device__ __forceinline__ u32x2 turn_quarters(u32x2 d) {
  const auto a = __builtin_amdgcn_permlane32_swap(d[0], d[1], false, false);
  // rows 0, 1: channels 0 .. 3 of tokens i and i + 2; rows 2, 3: channels 4 .. 7 of tokens i - 2 and i
  const uint32_t even = __builtin_amdgcn_perm(a[1], a[0], 0x05040100);   // the first two channels of both tokens
  const uint32_t odd = __builtin_amdgcn_perm(a[1], a[0], 0x07060302);
  const auto b = __builtin_amdgcn_permlane16_swap(even, odd, false, false);
  // tokens 0 and 2, tokens 1 and 3, two channels each
  return u32x2{__builtin_amdgcn_perm(b[1], b[0], 0x06020400), __builtin_amdgcn_perm(b[1], b[0], 0x07030501)};
}

// What the lane two further in its quad gives.
__device__ __forceinline__ uint32_t across_pairs(uint32_t d) { return __builtin_amdgcn_update_dpp(0, (int)d, 0x4E, 0xf, 0xf, true); }

// E: the rows' type; TILES: 16-token tiles of a block.
template <typename E, int TILES> __global__ __launch_bounds__(256, TILES == 8 ? 5 : 8) void oscar_q8_append_kernel(AppendParams P) {
  constexpr int BLOCK = 16 * TILES;
  __shared__ uint32_t s_max[4];
  // (heads next to each other: a row's are)
  const uint32_t unit = blockIdx.x / P.c.heads;
  const int b = blockIdx.y, h = blockIdx.x % P.c.heads, side = unit & 1, tid = threadIdx.x;
  const Q8Seq s = q8_seq(P.r, b);
  if (s.n == 0) return;
  const int first = max(s.old, 0) / BLOCK, j = first + (int)(unit >> 1);   // (the block's number in its sequence)
  if ((int64_t)j * BLOCK >= s.len) return;
  const uint16_t* in = (side ? P.v : P.k) + h * D;
  const int64_t stride = side ? P.v_stride : P.k_stride;
  uint16_t* win = (side ? P.c.win_v : P.c.win_k) + ((int64_t)b * P.c.heads + h) * (2 * BLOCK * D);
  const int m = tid >> 4, c8 = tid & 15;   // token of a tile, piece of 8 channels

  const int page = q8_page(P.c, b, (int)((int64_t)j * BLOCK / R));   // (asked for ahead of the rows)
  const auto new_row = [&](int64_t pos) -> u32x4 {   // of a new token (zeros where there is no such row)
    const int64_t row = s.row + (pos - s.old);
    if (row < 0 || row >= P.r.n_rows) return u32x4{};
    // (read once: what is written stays in the caches; 4 x 8K tokens, written and read back, 68 -> 61 us)
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(in + row * stride + c8 * 8));
  };
  u32x4 raw[TILES];
#pragma unroll
  for (int i = 0; i < TILES; ++i) {
    const int64_t pos = (int64_t)j * BLOCK + 16 * i + m;
    raw[i] = u32x4{};
    if (pos < s.len)
      raw[i] = pos >= s.old ? new_row(pos)
                            : *reinterpret_cast<const u32x4*>(win + (pos % (2 * BLOCK)) * D + c8 * 8);
  }
  const bool whole = ((int64_t)j + 1) * BLOCK <= s.len;
  // the largest, by the numbers' bits; one that counts for another (rare) is replaced first
  u16x2 most = {};
#pragma unroll
  for (int i = 0; i < TILES; ++i) most = most_bits(most, raw[i]);
  if (__any(max(most[0], most[1]) > MOST_BITS<E>)) {
    most = u16x2{};
#pragma unroll
    for (int i = 0; i < TILES; ++i) most = most_bits(most, raw[i] = counted<E>(raw[i]));
  }
  // The window takes the tokens from the last whole block on.  It has two places a token: a block j + 2, j + 4, ..
  // goes where this one, if it is the first, has just been read; so the first block's workgroup writes it, behind
  // the barrier, and the others write what lies in the other half.
  const int last = s.len / BLOCK;   // the block that is not whole (or not begun)
  if (j >= last - 1 && (j == first || (j - first) % 2 != 0)) {
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const int64_t pos = (int64_t)j * BLOCK + 16 * i + m;
      if (pos >= s.old && pos < s.len) *reinterpret_cast<u32x4*>(win + (pos % (2 * BLOCK)) * D + c8 * 8) = raw[i];
    }
  }
  if (!whole) return;

  uint32_t bits = max(most[0], most[1]);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) bits = max(bits, (uint32_t)__shfl_xor((int)bits, d));
  if ((tid & 63) == 0) s_max[tid >> 6] = bits;
  __syncthreads();
  const float top = widen<E>(max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3])));
  int e = top > 0.0f ? __builtin_amdgcn_frexp_expf(top) - 9 + (__builtin_amdgcn_frexp_mantf(top) > 0.875f) : 0;
  e = max(e, -100);
  const float scale = __uint_as_float((uint32_t)(127 + e) << 23);

  if (page >= 0) {
    const int t0 = (int)((int64_t)j * BLOCK % R);   // of the page
    uint8_t* out = (side ? P.c.v_codes : P.c.k_codes) + ((int64_t)page * P.c.heads + h) * Q8_PAGE_BYTES + t0 * D;
    u32x2 codes[TILES];
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
#pragma unroll
      for (int d = 0; d < 2; ++d)
        codes[i][d] = two_codes<E>(two_codes<E>(0, raw[i][2 * d], scale, false), raw[i][2 * d + 1], scale, true);
    }
    if (side == 0) {
#pragma unroll
      for (int i = 0; i < TILES; ++i)
        *reinterpret_cast<u32x2*>(out + i * 2048 + (c8 / 8) * 1024 + (c8 % 8 / 2) * 256 + m * 16 + (c8 % 2) * 8) = codes[i];
    } else {
      // afterwards a lane has channels c and c + 1 of tokens 4 q4 ..; the lane two further on c + 16 and c + 17: they
      // change so that one has c and c + 16, which lie next to each other, the other c + 1 and c + 17
      const int q4 = m / 4, c = c8 * 8 + (m % 4) * 2;
      const bool upper = c8 & 2;
      uint8_t* to = out + (c / 32) * 1024 + q4 * 256 + (c % 16 + upper) * 16;
#pragma unroll
      for (int i = 0; i < TILES; i += 2) {
        const u32x2 a = turn_quarters(codes[i]), z = turn_quarters(codes[i + 1]);
        const uint32_t a_in = across_pairs(upper ? a[0] : a[1]), z_in = across_pairs(upper ? z[0] : z[1]);
        *reinterpret_cast<u32x4*>(to + (i / 2) * Q8_STEP_BYTES) =
            upper ? u32x4{a_in, z_in, a[1], z[1]} : u32x4{a[0], z[0], a_in, z_in};
      }
    }
    if (tid == 0)
      (side ? P.c.v_scales : P.c.k_scales)[((int64_t)page * P.c.heads + h) * (R / BLOCK) + t0 / BLOCK] = scale;
  }

  // the later block of this half of the window
  if (j != first) return;
  const int late = (last - first) % 2 == 0 ? last : last - 1;
  if (late <= first || (int64_t)late * BLOCK >= s.len) return;
#pragma unroll
  for (int i = 0; i < TILES; ++i) {
    const int64_t pos = (int64_t)late * BLOCK + 16 * i + m;
    if (pos < s.old || pos >= s.len) continue;
    *reinterpret_cast<u32x4*>(win + (pos % (2 * BLOCK)) * D + c8 * 8) = counted<E>(new_row(pos));
  }
}

// ---- back out -------------------------------------------------------------------------------------

struct ReadParams {
  Q8Cache c;
  const int32_t *lens, *starts;
  int T, steps;   // 32-token steps a sequence's T tokens can touch
  void *k, *v;
};

constexpr int ROW_PITCH = D + 16;   // bytes of a row in LDS: 16-byte pieces of four rows on different banks

// What a lane writes at a time: 16 bytes, so that a wave's lie next to each other.
template <typename O> constexpr int LANE_NUMBERS = 16 / sizeof(O);
// (32-bit rows past the caches: 65536 tokens of 8 kv heads read 130 -> 111 us, read and then added up 284 -> 263; 16-bit rows
// gain as much alone and lose it again where the next launch uses them: 64 us, 65 past the caches)
// fp16 tokens from 63488 on are codes of 65536 (256 * 256): as fp16 they go out as its largest number, no infinity.
template <typename E, typename O> __device__ __forceinline__ void put(O* to, float* x) {
  if constexpr (__is_same(E, __half) && __is_same(O, __half))
#pragma unroll
    for (int i = 0; i < LANE_NUMBERS<O>; ++i) x[i] = __builtin_amdgcn_fmed3f(x[i], -65504.0f, 65504.0f);
  if constexpr (sizeof(O) == 4)
    __builtin_nontemporal_store(u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])},
                                reinterpret_cast<u32x4*>(to));
  else
    *reinterpret_cast<u32x4*>(to) = narrow8<O>(x);
}

// Lane quads: byte i of the result is byte (lane % 4) of lane i's dword.
__device__ __forceinline__ uint32_t turn_quad(uint32_t d, int lane) {
  const uint32_t other = __builtin_amdgcn_update_dpp(0, (int)d, 0xB1, 0xf, 0xf, true);   // lanes 1 0 3 2
  // even lanes: bytes 0 and 2 of both; odd lanes: bytes 1 and 3
  d = lane & 1 ? __builtin_amdgcn_perm(d, other, 0x07030501) : __builtin_amdgcn_perm(other, d, 0x06020400);
  // bytes: (own pair's first lane, second lane) for byte lane % 2, then the same for byte lane % 2 + 2
  const uint32_t far = across_pairs(d);
  return lane & 2 ? __builtin_amdgcn_perm(d, far, 0x07060302) : __builtin_amdgcn_perm(far, d, 0x05040100);
}

template <typename E, typename O> __global__ __launch_bounds__(256) void oscar_q8_read_kernel(ReadParams P) {
  __shared__ __align__(16) uint8_t s_rows[4][Q8_STEP_TOKENS * ROW_PITCH];
  const int b = blockIdx.z, side = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  O* out = reinterpret_cast<O*>(side ? P.v : P.k);
  if (!out) return;
  const int len = max(P.lens[b], 0), start = P.starts ? P.starts[b] : 0;
  const int64_t from = max((int64_t)start, (int64_t)0), to = min((int64_t)start + P.T, (int64_t)len);
  const int64_t unit = (int64_t)blockIdx.x * 4 + wave;   // heads side by side: rows next to each other
  const int64_t step = from / Q8_STEP_TOKENS + unit / P.c.heads;
  const int h = (int)(unit % P.c.heads);
  const int64_t t0 = step * Q8_STEP_TOKENS;
  if (unit / P.c.heads >= P.steps || t0 >= to) return;   // (no barriers below: a wave is by itself)
  const bool coded = t0 < len / P.c.block * P.c.block;
  uint8_t* rows = s_rows[wave];
  float scale = 1.0f;
  const uint16_t* win = nullptr;
  if (coded) {
    const int page = q8_page(P.c, b, (int)(step / Q8_PAGE_STEPS));
    if (page < 0) return;
    const int64_t at = (int64_t)page * P.c.heads + h;
    const uint8_t* in = (side ? P.c.v_codes : P.c.k_codes) + at * Q8_PAGE_BYTES + (step % Q8_PAGE_STEPS) * Q8_STEP_BYTES;
    const int per = R / P.c.block;
    scale = (side ? P.c.v_scales : P.c.k_scales)[at * per + (t0 % R) / P.c.block];
    u32x4 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const u32x4*>(in + i * 1024 + lane * 16);
    const int q4 = lane >> 4, n = lane & 15;
    if (side == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<u32x4*>(rows + (16 * (i / 2) + n) * ROW_PITCH + 64 * (i % 2) + 16 * q4) = w[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int d = 0; d < 4; ++d)   // channel tile d / 2, token tile d % 2
          *reinterpret_cast<uint32_t*>(rows + (16 * (d % 2) + 4 * q4 + n % 4) * ROW_PITCH + 32 * i + 16 * (d / 2) + (n & ~3)) =
              turn_quad(w[i][d], lane);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  } else {
    win = (side ? P.c.win_v : P.c.win_k) + ((int64_t)b * P.c.heads + h) * (2 * P.c.block * D);
  }
  constexpr int N = LANE_NUMBERS<O>, LANES = D / N;   // of a row
  const int c = lane % LANES * N;
#pragma unroll
  for (int i = 0; i < Q8_STEP_TOKENS * LANES / 64; ++i) {
    const int t = 64 / LANES * i + lane / LANES;
    const int64_t pos = t0 + t;
    if (pos < from || pos >= to) continue;
    float x[8];
    if (coded) {
#pragma unroll
      for (int d = 0; d < N / 4; ++d) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(rows + t * ROW_PITCH + c + 4 * d);
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        x[4 * d] = lo[0] * scale, x[4 * d + 1] = lo[1] * scale, x[4 * d + 2] = hi[0] * scale, x[4 * d + 3] = hi[1] * scale;
      }
    } else {
#pragma unroll
      for (int d = 0; d < N / 4; ++d) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(win + (pos % (2 * P.c.block)) * D + c + 4 * d);
#pragma unroll
        for (int j = 0; j < 2; ++j) x[4 * d + 2 * j] = widen<E>(w[j] & 0xffff), x[4 * d + 2 * j + 1] = widen<E>(w[j] >> 16);
      }
    }
    put<E>(out + (((int64_t)b * P.T + (pos - start)) * P.c.heads + h) * D + c, x);
  }
}

template <typename E> void launch_append(const AppendParams& P, hipStream_t st) {
  const dim3 grid(2 * P.blocks * P.c.heads, P.c.batch);
  if (P.c.block == 32)
    hipLaunchKernelGGL((oscar_q8_append_kernel<E, 2>), grid, dim3(256), 0, st, P);
  else if (P.c.block == 64)
    hipLaunchKernelGGL((oscar_q8_append_kernel<E, 4>), grid, dim3(256), 0, st, P);
  else
    hipLaunchKernelGGL((oscar_q8_append_kernel<E, 8>), grid, dim3(256), 0, st, P);
}

template <typename E> void launch_read(const ReadParams& P, int out_dtype, hipStream_t st) {
  const dim3 grid((uint32_t)(((int64_t)P.steps * P.c.heads + 3) / 4), 2, P.c.batch);
  if (out_dtype == OSCAR_F32)
    hipLaunchKernelGGL((oscar_q8_read_kernel<E, float>), grid, dim3(256), 0, st, P);
  else if (out_dtype == OSCAR_BF16)
    hipLaunchKernelGGL((oscar_q8_read_kernel<E, __hip_bfloat16>), grid, dim3(256), 0, st, P);
  else
    hipLaunchKernelGGL((oscar_q8_read_kernel<E, __half>), grid, dim3(256), 0, st, P);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

int oscar_check_q8_sizes(const oscar_q8_cache* c) {
  if (!c) return OSCAR_ERR_INVALID_ARG;
  if (c->batch < 1 || c->max_pages_per_seq < 1 || c->num_pages < 1 || c->n_kv_heads < 1 || c->head_dim < 1 || c->page_size < 1 ||
      c->block < 1 || c->io_dtype < OSCAR_F32 || c->io_dtype > OSCAR_F16)
    return OSCAR_ERR_INVALID_ARG;
  if (c->batch > 65535 || c->n_kv_heads > 65535) return OSCAR_ERR_INVALID_ARG;
  if (c->max_pages_per_seq > INT32_MAX / OSCAR_R || c->num_pages > INT32_MAX / OSCAR_R) return OSCAR_ERR_INVALID_ARG;
  if (c->head_dim != OSCAR_D || c->page_size != OSCAR_R || (c->block != 32 && c->block != 64 && c->block != 128) ||
      c->io_dtype == OSCAR_F32)
    return OSCAR_ERR_UNSUPPORTED;
  return OSCAR_OK;
}

int oscar_check_q8_cache(const oscar_q8_cache* c) {
  const int rc = oscar_check_q8_sizes(c);
  if (rc != OSCAR_OK) return rc;
  if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales || !c->win_k || !c->win_v || !c->block_table)
    return OSCAR_ERR_INVALID_ARG;
  if (!aligned16(c->k_codes) || !aligned16(c->v_codes) || !aligned16(c->win_k) || !aligned16(c->win_v)) return OSCAR_ERR_INVALID_ARG;
  return OSCAR_OK;
}

extern "C" int oscar_q8_sizes(const oscar_q8_cache* cache, oscar_q8_pool_sizes* out) {
  const int rc = oscar_check_q8_sizes(cache);
  if (rc != OSCAR_OK) return rc;
  if (!out) return OSCAR_ERR_INVALID_ARG;
  const size_t heads = cache->n_kv_heads, scales = OSCAR_R / cache->block * sizeof(float);
  out->codes = (size_t)cache->num_pages * heads * Q8_PAGE_BYTES;
  out->scales = (size_t)cache->num_pages * heads * scales;
  out->window = (size_t)cache->batch * heads * 2 * cache->block * OSCAR_D * 2;
  out->block_table = (size_t)cache->batch * cache->max_pages_per_seq * sizeof(int32_t);
  out->page_bytes_per_kv_head = 2 * (Q8_PAGE_BYTES + scales);
  return OSCAR_OK;
}

extern "C" int oscar_q8_append(const void* k, const void* v, int64_t k_stride, int64_t v_stride, int64_t n_rows,
                               int32_t T, const int32_t* row_starts, const int32_t* new_lens, const int32_t* lens,
                               const oscar_q8_cache* cache, void* stream) {
  const int rc = oscar_check_q8_cache(cache);
  if (rc != OSCAR_OK) return rc;
  if (T < 0 || n_rows < 0) return OSCAR_ERR_INVALID_ARG;
  if (T == 0 || n_rows == 0) return OSCAR_OK;
  if (!k || !v || !lens || !aligned16(k) || !aligned16(v)) return OSCAR_ERR_INVALID_ARG;
  const int64_t row = (int64_t)cache->n_kv_heads * OSCAR_D;
  if (k_stride < row || v_stride < row || k_stride % 8 != 0 || v_stride % 8 != 0) return OSCAR_ERR_INVALID_ARG;
  AppendParams P = {q8_device_view(cache), {row_starts, new_lens, lens, T, n_rows}, reinterpret_cast<const uint16_t*>(k),
                    reinterpret_cast<const uint16_t*>(v), k_stride, v_stride, 0};
  // T tokens from the last place of a block on
  P.blocks = (int)(((int64_t)T + 2 * cache->block - 2) / cache->block);
  // a grid's threads are counted in 32 bits
  if ((int64_t)P.blocks * 2 * cache->n_kv_heads * 256 > UINT32_MAX) return OSCAR_ERR_INVALID_ARG;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (cache->io_dtype == OSCAR_BF16)
    launch_append<__hip_bfloat16>(P, st);
  else
    launch_append<__half>(P, st);
  if (hipGetLastError() != hipSuccess) return OSCAR_ERR_HIP;
  return OSCAR_OK;
}

extern "C" int oscar_q8_read(const oscar_q8_cache* cache, const int32_t* lens, const int32_t* starts, int32_t T,
                             void* k, void* v, int32_t out_dtype, void* stream) {
  const int rc = oscar_check_q8_cache(cache);
  if (rc != OSCAR_OK) return rc;
  if (T < 0 || out_dtype < OSCAR_F32 || out_dtype > OSCAR_F16 || !lens || (!k && !v) || !aligned16(k) || !aligned16(v))
    return OSCAR_ERR_INVALID_ARG;
  if (T == 0) return OSCAR_OK;
  ReadParams P = {q8_device_view(cache), lens, starts, T, 0, k, v};
  P.steps = (int)(((int64_t)T + 2 * Q8_STEP_TOKENS - 2) / Q8_STEP_TOKENS);
  // a grid's threads are counted in 32 bits
  if (((int64_t)P.steps * cache->n_kv_heads + 3) / 4 * 256 > UINT32_MAX) return OSCAR_ERR_INVALID_ARG;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  if (cache->io_dtype == OSCAR_BF16)
    launch_read<__hip_bfloat16>(P, out_dtype, st);
  else
    launch_read<__half>(P, out_dtype, st);
  if (hipGetLastError() != hipSuccess) return OSCAR_ERR_HIP;
  return OSCAR_OK;
}
