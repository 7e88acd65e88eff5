// Keys and values of a served model in a paged cache of 4-bit codes, and attention over it.
//
// A row (the key or the value of one token and kv head, dim values) is quantised on the min-max
// grid of the weights, 16 levels: after an optional Hadamard transform r = H v / sqrt(dim) (which
// spreads a strong channel over the row; queries take the same transform, so that products do not
// change, and outputs its inverse, H again),
//   scale = (max(0, r) - min(0, r)) / 15 rounded up to bf16 (at least 2^-100),
//   zero = rint(-min(0, r) / scale), code = clamp(rint(r / scale) + zero, 0, 15).
// Layout: codes [page][kv head][key, value][words of a page], eight codes to a word, low bits
// first; a key row is dim / 8 consecutive words, value rows are interleaved four tokens at a time
// ([token / 4][word][token % 4]) so that a lane's load brings it four tokens of its channels.
// params [page][kv head][key, value][token]: scale (bf16, upper half) and zero (lower half).
#include <cmath>
#include <type_traits>

#include "kq_common.hpp"
#include "kq_fwht.hpp"

namespace kq {
namespace {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint16_t f32_bf16(float v) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

// The chunk of 8 channels that lane n of each 16 holds: the chunk 4 further on is the mirrored lane of
// 8, so that every stage between chunks is one multiply-add.
__device__ __forceinline__ int chunk_of(int n) { return n ^ ((n & 4) ? 3 : 0); }

// ---- append --------------------------------------------------------------------------------------
struct AppendArgs {
  const void *k, *v;
  int64_t ldk, ldv, n_tokens;
  int n_kv, page_log;
  int64_t n_slots;
  const int64_t* slots;
  uint32_t *codes, *params;
  int rotate;
  double norm;
  float *k_hat, *v_hat;
};

// What a lane has found of its row: the codes of its eight values, the row's scale, zero and whether
// all of it is finite.
struct RowGrid {
  uint32_t word;
  float scale, zero;
  bool bad;
};

// The grid in fp64: the transform is exact to 2^-52, so that a code depends on the row alone and not
// on the order of the sums.
template <int LPR>
__device__ __forceinline__ RowGrid row_grid(const float (&x)[8], int chunk, int rotate, double norm) {
  double r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = x[i];
  if (rotate) {
#pragma unroll
    for (int s = 1; s < 8; s <<= 1)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (!(i & s)) {
          const double a = r[i], b = r[i + s];
          r[i] = a + b, r[i + s] = a - b;
        }
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double p = __shfl_xor(r[i], o == 4 ? 7 : o);
        r[i] = (chunk & o) ? p - r[i] : r[i] + p;
      }
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] *= norm;
  }
  double lo = 0.0, hi = 0.0;
  int bad = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fmin(lo, r[i]), hi = fmax(hi, r[i]);
    bad |= !(fabs(r[i]) <= 3.0e38);  // NaN, infinities, and values whose grid bf16 cannot hold
  }
#pragma unroll
  for (int o = 1; o < LPR; o <<= 1) {
    lo = fmin(lo, __shfl_xor(lo, o)), hi = fmax(hi, __shfl_xor(hi, o));
    bad |= __shfl_xor(bad, o);
  }
  const double wide = fmax((hi - lo) / 15.0, 0x1p-100);
  // up to bf16: 45 of the 52 bits of the fraction go
  const uint64_t up = (__builtin_bit_cast(uint64_t, wide) + ((uint64_t(1) << 45) - 1)) &
                      ~((uint64_t(1) << 45) - 1);
  const double scale = __builtin_bit_cast(double, up), inv = 1.0 / scale;
  const double zero = fmin(rint(-lo / scale), 15.0);
  RowGrid g{0, float(scale), float(zero), bad != 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double t = r[i] * inv;  // good to 2^-51: rint(t) is rint(r / scale) unless t is next to a
    double n = rint(t);           // half, where the quotient itself decides
    if (fabs(fabs(t - n) - 0.5) < 1e-12) n = rint(r[i] / scale);
    const double c = bad ? 0.0 : fmin(fmax(n + zero, 0.0), 15.0);
    g.word |= uint32_t(int(c)) << (4 * i);
  }
  return g;
}

// dim / 8 lanes take a row, eight values each. The grid is worked out in fp32 and kept where fp32
// must agree with fp64, which settles the rest (some rows of 100). The transform before its norm, f,
// has log2(D) <= 7 stages; each rounds by at most 2^-24 of its result in the 2-norm and all later ones
// scale that as they scale the result, so |error of f|_2 <= 7 2^-24 |f|_2. With t = r / scale, whose
// range is 14.8 to 15,
//   |error of t| < 4.2e-7 |t|_2 + 3 2^-24 15: halves are kept clear by 4.24e-7 |t|_2 + 4e-6;
//   the range's error is twice that of a value, |t|_2 steps of a 24-bit fraction and some for the
//     products after it: where the scale is cut, 16 of those bits, |t|_2 + 8 steps are kept clear.
// 16000 tokens of 8 heads of 128 (213 MB with what the cache holds): 53 us, 4.0 TB/s; all of it in fp64
// was bound by that arithmetic, 72 us.
template <typename T, int DIM>
__global__ __launch_bounds__(256) void cache_append(AppendArgs A) {
  constexpr int LPR = DIM / 8, RPW = 256 / LPR;  // lanes per row, rows per workgroup
  const int l = threadIdx.x % LPR;
  const int chunk = chunk_of(l);
  const int64_t row = workgroup() * RPW + threadIdx.x / LPR;  // token, head, key or value
  const int64_t rows = A.n_tokens * A.n_kv * 2;
  if (row >= rows) return;  // (whole groups of LPR lanes)
  const int part = int(row & 1);
  const uint32_t th = uint32_t(row >> 1), token = th / uint32_t(A.n_kv);  // (at most 2^31 of them)
  const int head = int(th - token * uint32_t(A.n_kv));
  const int64_t slot = A.slots[token];
  if (slot < 0 || slot >= A.n_slots) return;
  const T* src = static_cast<const T*>(part ? A.v : A.k) +
                 int64_t(token) * (part ? A.ldv : A.ldk) + int64_t(head) * DIM + chunk * 8;
  float x[8], f[8];
  if constexpr (sizeof(T) == 2) {
    const uint4 w = *reinterpret_cast<const uint4*>(src);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const float4 w = *reinterpret_cast<const float4*>(src + i);
      x[i] = w.x, x[i + 1] = w.y, x[i + 2] = w.z, x[i + 3] = w.w;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = x[i];
  float norm = 1.f, sign = 1.f;
  if (A.rotate) {
    hadamard_reg<8>(f);
    stage_lane1(f, (chunk & 1) ? -1.f : 1.f);
    stage_lane2(f, (chunk & 2) ? -1.f : 1.f);
    stage_mirror8(f, (chunk & 4) ? -1.f : 1.f);
    if constexpr (LPR == 16) stage_lane8(f, (chunk & 8) ? -1.f : 1.f);
    norm = float(A.norm), sign = (__popc(unsigned(chunk)) & 1) ? -1.f : 1.f;
  }
  float lo = f[0], hi = f[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) lo = fminf(lo, f[i]), hi = fmaxf(hi, f[i]);
  const float least = sign < 0.f ? -hi : lo, most = sign < 0.f ? -lo : hi;
  lo = fminf(least, 0.f), hi = fmaxf(most, 0.f);
  auto join = [&](auto other) {
    lo = fminf(lo, other(lo)), hi = fmaxf(hi, other(hi));
  };
  join([](float v) { return dpp_mov<0xB1>(v); });
  join([](float v) { return dpp_mov<0x4E>(v); });
  join([](float v) { return dpp_mov<0x141>(v); });
  if constexpr (LPR == 16) join([](float v) { return dpp_mov<0x128>(v); });
  const float range = hi - lo, step = range * (norm / 15.f);
  const uint32_t bits = __float_as_uint(fmaxf(step, 0x1p-100f));
  RowGrid g;
  g.scale = __uint_as_float((bits + 0xFFFFu) & 0xFFFF0000u);
  const float inv = norm / g.scale, to = inv * sign, z = -lo * inv;
  g.zero = fminf(rintf(z), 15.f), g.bad = false, g.word = 0;
  float far = fabsf(z - rintf(z)), sum = 0.f;  // from the next whole number; |t|_2 squared
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = f[i] * to, n = rintf(t);
    far = fmaxf(far, fabsf(t - n)), sum = fmaf(t, t, sum);
    const float c = fminf(fmaxf(n + g.zero, 0.f), 15.f);
    g.word |= uint32_t(int(c)) << (4 * i);
  }
  auto row_of = [&](auto other) { far = fmaxf(far, other(far)), sum += other(sum); };
  row_of([](float v) { return dpp_mov<0xB1>(v); });
  row_of([](float v) { return dpp_mov<0x4E>(v); });
  row_of([](float v) { return dpp_mov<0x141>(v); });
  if constexpr (LPR == 16) row_of([](float v) { return dpp_mov<0x128>(v); });
  // (a value that is not finite makes the range infinite or the sum NaN; step below the least scale
  // is not cut)
  const float low = float(bits & 0xFFFFu), clear = fminf(low, 65536.f - low) - 8.f;
  const float half = 0.5f - 4e-6f - far;
  const bool sure = half > 0.f && half * half > 1.8e-13f * sum && range <= 3.0e38f &&
                    (step < 0x1.fp-101f || (clear > 0.f && clear * clear > sum));
  if (!sure) g = row_grid<LPR>(x, chunk, A.rotate, A.norm);
  // a row with a value that is not finite reads as NaN
  if (g.bad) g.scale = __uint_as_float(0x7FC00000u);
  const int64_t p = slot >> A.page_log, off = slot & ((int64_t(1) << A.page_log) - 1);
  const int64_t ph = (p * A.n_kv + head) * 2 + part;
  const int64_t at = part ? ((off >> 2) * LPR + chunk) * 4 + (off & 3) : off * LPR + chunk;
  A.codes[((ph << A.page_log) * LPR) + at] = g.word;
  if (l == 0)
    A.params[(ph << A.page_log) + off] =
        __float_as_uint(g.scale) | (g.bad ? 0u : uint32_t(int(g.zero)));
  float* out = part ? A.v_hat : A.k_hat;
  if (out) {
    out += int64_t(th) * DIM + chunk * 8;
    float hat[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) hat[i] = g.scale * (float((g.word >> (4 * i)) & 15u) - g.zero);
    *reinterpret_cast<float4*>(out) = make_float4(hat[0], hat[1], hat[2], hat[3]);
    *reinterpret_cast<float4*>(out + 4) = make_float4(hat[4], hat[5], hat[6], hat[7]);
  }
}

// ---- attention -----------------------------------------------------------------------------------
// For one sequence and kv head, the new tokens' queries of the heads that share it are rows: row
// i G + g is token i, head g of G. A wave takes 16 MQ rows and walks a range of the cached tokens, 32
// at a time, one pass with a running maximum and sums. The four waves of a workgroup
//   BY_ROWS (prompts): take different rows and the same tokens; each ends with its own rows;
//   otherwise (few rows: decoding): take the same rows and tokens in turn, and meet in LDS at the end.
// Beside that a range of tokens is split over workgroups where rows are few; attention_join ends that.
//   scores   S[token][row] = K q on v_mfma_f32_16x16x32_f16, twice 16 tokens: a lane spreads the
//            codes of its token and channels straight from the loaded words. A code left at bit 0
//            or 4 of its half word is the subnormal fp16 c 2^-24 or c 2^-20, so a pair of codes
//            costs one AND (and every second word a shift); the power of 16 between the two is
//            inside q. S = s_t (sum c q - z_t sum q).
//   weights  p = 2^(S - m) with m a reference that follows the running maximum only when that
//            leaves it by more than 2^7, so that most tiles rescale nothing and compare without
//            crossing lanes. The weight that meets the value codes is p s_t / sigma as fp16, sigma
//            following the row's largest value scale the same way.
//   outputs  O[row][channel] += (p s) c: the lane that held S for a row and four tokens of either
//            half holds its weights for the same tokens as the A operand (the order of tokens in a
//            sum is free), so nothing crosses lanes; sum (p s) z beside it.
// fp16 for q (2^-11), for the weights (2^-11, and never coarser than 2^-25 of the row's largest value
// scale); everything summed in fp32; outputs bf16.
struct AttnArgs {
  const uint16_t* q;
  int64_t ldq, n_tokens;
  int n_heads, n_kv, group;
  const uint32_t *codes, *params;
  int64_t n_pages;
  int page_log;
  const int* table;
  int64_t ldt;
  int table_pages;
  const int* lengths;
  const int* starts;  // null: token b is sequence b
  float scale;        // of the scores, times log2(e)
  int rotate, fill;
  int tiles, splits;
  uint16_t* out;
  int64_t ldo;
  bool wide;          // 16-byte stores of outputs
  float *part, *ml;   // splits > 1: [split][token][head][dim], and maximum and sum
};

// lane + 64 e of a row of DIM = 64 or 128 values: H x / sqrt(DIM)
template <int DIM>
__device__ __forceinline__ void rotate_row(float (&x)[2], int lane) {
  hadamard_lanes<2>(x, lane);
  if constexpr (DIM == 128) {
    const float a = x[0], b = x[1];
    x[0] = a + b, x[1] = a - b;
  }
  x[0] *= DIM == 128 ? 0.08838834764831845f : 0.125f;
  x[1] *= 0.08838834764831845f;
}

template <int DIM>
__device__ __forceinline__ void store_row(uint16_t* o, float (&x)[2], int lane, int rotate) {
  if (rotate) rotate_row<DIM>(x, lane);
  o[lane] = f32_bf16(x[0]);
  if constexpr (DIM == 128) o[lane + 64] = f32_bf16(x[1]);
}

__device__ __forceinline__ f32x4_t mfma16(u32x4_t a, u32x4_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a),
                                                __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

#define KQ_LDS(p) ((__attribute__((address_space(3))) void*)(p))
template <int N>
__device__ __forceinline__ void wait_vm() {  // s_waitcnt vmcnt(N), the other counters free
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

// What a wave keeps in LDS of 32 tokens, in two halves of 16: for each lane the words of its key row
// and of its value channels as it wants them (16 bytes a lane and load, one behind another), and the
// parameters of 16 keys and 16 values. The loads go straight there, DEPTH tiles ahead: registers for
// a second tile left one wave less per SIMD and a single tile of each wave on its way: 156 us for 48
// sequences of up to 16384 tokens, 64 heads, where it takes 120 now, 4.1 TB/s of the cache (a copy
// reaches 4.7, a sum over what was read 4.0).
constexpr int DEPTH = 4;
constexpr float NONE = -1e30f;
constexpr int tile_words(int dim) { return 2 * (64 * (dim / 32) + 256 + 64); }

template <int DIM, int MQ, bool BY_ROWS>
__global__ __launch_bounds__(256, 2) void cache_attention(AttnArgs A) {
  constexpr int NJ = DIM / 32;       // words of a key row a lane takes, matrix steps per score
  constexpr int ND = DIM / 16;       // output blocks of 16 channels
  constexpr int WPR = DIM / 8;       // words per row
  constexpr int ROWS = 16 * MQ, TILE = BY_ROWS ? 4 * ROWS : ROWS, LD = DIM + 4;
  constexpr int STEP = BY_ROWS ? 32 : 128;  // tokens from one of a wave's tiles to the next
  constexpr int TW = tile_words(DIM), HALF = TW / 2, AT_V = 64 * NJ, AT_P = AT_V + 256;
  // the waves' tiles [wave][DEPTH][TW]; at the end [wave][row][LD] and [wave][row][2]
  extern __shared__ __attribute__((aligned(16))) float sm[];
  float* sml = sm + 4 * ROWS * LD;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g4 = lane >> 4;
  const int b = blockIdx.y, h = blockIdx.x;
  const int split = blockIdx.z % A.splits;
  const int nt = int(A.n_tokens);
  int q0 = b, q1 = b + 1;
  if (A.starts) {
    q0 = __builtin_amdgcn_readfirstlane(A.starts[b]);
    q1 = __builtin_amdgcn_readfirstlane(A.starts[b + 1]);
    q0 = q0 < 0 ? 0 : q0 > nt ? nt : q0;
    q1 = q1 < q0 ? q0 : q1 > nt ? nt : q1;
    if (A.fill) {  // tokens before the first sequence and behind the last one, dealt to all workgroups
      const int s0 = A.starts[0], s1 = A.starts[gridDim.y];
      const int head = s0 < 0 ? 0 : s0 > nt ? nt : s0, tail = s1 < head ? head : s1 > nt ? nt : s1;
      const int64_t all = int64_t(gridDim.y) * gridDim.z;  // (may pass 2^31)
      const int width = A.group * DIM;
      for (int64_t k = b + int64_t(gridDim.y) * blockIdx.z; k < head + nt - tail; k += all) {
        uint16_t* const out = A.out + (k < head ? k : k - head + tail) * A.ldo + int64_t(h) * width;
        for (int e = tid; e < width; e += 256) out[e] = 0;
      }
    }
  }
  const int nq = q1 - q0, G = A.group, nrows = nq * G;
  int len = __builtin_amdgcn_readfirstlane(A.lengths[b]);
  const int most = A.table_pages << A.page_log;
  len = len < 0 ? 0 : len > most ? most : len;
  const int* table = A.table + int64_t(b) * A.ldt;
  const int page_mask = (1 << A.page_log) - 1;
  // later rows see more tokens: they go first, of all sequences (by sequences, the last ones of a long
  // sequence late in the grid ran alone at the end: 244 us in a trace for prompts of 2048 to 274 tokens
  // and 32 heads, 170 this way; strictly by the tokens that rows see it was 181; not traced, a call of
  // the present kernel takes 162)
  const int tiles = (nrows + TILE - 1) / TILE;
  for (int tile = tiles - 1 - int(blockIdx.z / A.splits); tile >= 0; tile -= A.tiles) {
    const int row0 = tile * TILE + (BY_ROWS ? wave * ROWS : 0);
    if (BY_ROWS && row0 >= nrows) continue;
    const int end_row = row0 + ROWS < nrows ? row0 + ROWS : nrows;
    // tokens that the tile's first and last rows see
    const int see0 = len - nq + row0 / G + 1, see1 = len - nq + (end_row - 1) / G + 1;
    const int end = see1 > 0 ? see1 : 0;
    int chunk = (end + A.splits - 1) / A.splits;
    chunk = (chunk + 127) & ~127;
    const int beg_t = split * chunk, end_t = beg_t + chunk < end ? beg_t + chunk : end;

    // queries as the B operand: row n of each 16, channels 8 NJ g4 + 8 j + {0 4 1 5 2 6 3 7}, odd
    // pairs divided by 16; the whole row by a power of two
    u32x4_t qf[MQ][NJ];
    float qsum[MQ], qs[MQ];
    int see[MQ];
#pragma unroll
    for (int i = 0; i < MQ; ++i) {
      const int row = row0 + 16 * i + n < nrows ? row0 + 16 * i + n : nrows - 1;
      see[i] = len - nq + row / G + 1;
      const uint16_t* src = A.q + int64_t(q0 + row / G) * A.ldq + int64_t(h * G + row % G) * DIM;
      float x[8 * NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const u32x4_t w = *reinterpret_cast<const u32x4_t*>(src + 8 * (NJ * g4 + j));
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[8 * j + 2 * k] = __uint_as_float(w[k] << 16);
          x[8 * j + 2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        }
      }
      if (A.rotate) {
        hadamard_reg<8 * NJ>(x);
        stage_rows<8 * NJ, false>(x);
        stage_rows<8 * NJ, true>(x);
      }
      float mx = 0.f;
#pragma unroll
      for (int k = 0; k < 8 * NJ; ++k) mx = fmaxf(mx, fabsf(x[k]));
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const int e = int(__float_as_uint(mx) >> 23) - 127;
      const int ue = mx > 0.f && e < 128 ? (e < -90 ? -90 : e) - 5 : 0;  // largest to [2^5, 2^6)
      const float up = __uint_as_float(uint32_t(127 - ue) << 23);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        u32x4_t f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float lo = x[8 * j + k] * up, hi = x[8 * j + k + 4] * up;
          f16x2_t p = {_Float16(lo), _Float16(hi)};
          sum += float(p[0]) + float(p[1]);
          if (k & 1) p *= f16x2_t{_Float16(0.0625f), _Float16(0.0625f)};
          f[k] = __builtin_bit_cast(uint32_t, p);
        }
        qf[i][j] = f;
      }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      __builtin_amdgcn_sched_barrier(0);
      qsum[i] = sum * 0x1p-24f;
      qs[i] = A.scale * __uint_as_float(uint32_t(127 + ue) << 23) * 0x1p24f;
      if (A.rotate) qs[i] *= DIM == 128 ? 0.08838834764831845f : 0.125f;
    }

    f32x4_t acc[MQ][ND] = {};
    // the reference m of a row (NONE: it has seen no token), what is subtracted from its scores, and
    // how far above it they may be
    float m[MQ], ref[MQ], above[MQ], l[MQ], zs[MQ];
    // what the row's weights are divided by: within 2^7 of the largest value scale that it has seen (not
    // that the wave has: a later token's would take the weights of the rows before it)
    float sigma[MQ], sinv[MQ];
#pragma unroll
    for (int i = 0; i < MQ; ++i) {
      m[i] = NONE, ref[i] = 0.f, above[i] = -INFINITY;
      l[i] = zs[i] = sigma[i] = sinv[i] = 0.f;
    }

    // The pages of this wave's next 32 tiles, one of their halves of 16 a lane: read one by one, each
    // tile would wait for its page before it could ask for its codes. Tokens past the end: the last
    // ones again, masked below.
    const int first = beg_t + (BY_ROWS ? 0 : 32 * wave);
    int pages = 0, k0 = -32;
    const unsigned at_k = (n * WPR + g4 * NJ) * 4, at_v = (g4 * WPR + chunk_of(n & (WPR - 1))) * 16;
    const unsigned at_p = (n + ((lane & 16) << A.page_log >> 4)) * 4;  // keys, then values
    uint32_t* const ring = reinterpret_cast<uint32_t*>(sm) + wave * DEPTH * TW;
    auto token = [&](int t) { return t < end ? t : (end - 1) & ~15; };
    const int count = end_t > first ? (end_t - first + STEP - 1) / STEP : 0;
    unsigned bad = 0;  // two bits a tile under way: halves on pages that do not exist
    auto load = [&](int k) {  // this wave's tile k (past the end the last one, to a place of its own)
      const int place = k & (DEPTH - 1);
      k = k < count ? k : count - 1;
      if (k >= k0 + 32) {
        k0 = k;
        pages = table[token(first + STEP * (k + (lane >> 1)) + 16 * (lane & 1)) >> A.page_log];
      }
      uint32_t* const to = ring + place * TW;
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const int t = token(first + STEP * k + 16 * f);
        int p = __builtin_amdgcn_readlane(pages, 2 * (k - k0) + f);
        const unsigned bit = 1u << (2 * place + f);
        bad &= ~bit;
        if (p < 0 || p >= A.n_pages) p = 0, bad |= bit;
        const int64_t slot = (((int64_t(p) * A.n_kv + h) * 2) << A.page_log) + (t & page_mask);
        const auto codes = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint32_t*>(A.codes + slot * WPR), 0, 0x7FFFFFFF, 0x00027000);
        const auto params = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint32_t*>(A.params + slot), 0, 0x7FFFFFFF, 0x00027000);
        uint32_t* const half = to + f * HALF;
        if constexpr (NJ == 4) {
          __builtin_amdgcn_raw_ptr_buffer_load_lds(codes, KQ_LDS(half), 16, at_k, 0, 0, 0);
        } else {
          __builtin_amdgcn_raw_ptr_buffer_load_lds(codes, KQ_LDS(half), 4, at_k, 0, 0, 0);
          __builtin_amdgcn_raw_ptr_buffer_load_lds(codes, KQ_LDS(half + 64), 4, at_k, 4, 0, 0);
        }
        __builtin_amdgcn_raw_ptr_buffer_load_lds(codes, KQ_LDS(half + AT_V), 16, at_v,
                                                 (WPR * 4) << A.page_log, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(params, KQ_LDS(half + AT_P), 4, at_p, 0, 0, 0);
      }
    };
    constexpr int LOADS = 2 * (NJ == 4 ? 3 : 4);  // of a tile

    // CUT: some of the tokens do not count, or not for every row
    auto work = [&](int k, int t0, unsigned off, auto cut_c) {
      constexpr bool CUT = decltype(cut_c)::value;
      const uint32_t* const tile = ring + (k & (DEPTH - 1)) * TW;
      struct {
        uint32_t k[2][NJ], v[2][4], kp[2][4], vp[2][4];
      } T;
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const uint32_t* const half = tile + f * HALF;
        if constexpr (NJ == 4) {
          const u32x4_t w = *reinterpret_cast<const u32x4_t*>(half + 4 * lane);
          T.k[f][0] = w[0], T.k[f][1] = w[1], T.k[f][2] = w[2], T.k[f][3] = w[3];
        } else {
          T.k[f][0] = half[lane], T.k[f][1] = half[lane + 64];
        }
        const u32x4_t a = *reinterpret_cast<const u32x4_t*>(half + AT_P + 4 * g4);
        const u32x4_t c = *reinterpret_cast<const u32x4_t*>(half + AT_P + 16 + 4 * g4);
#pragma unroll
        for (int r = 0; r < 4; ++r) T.kp[f][r] = a[r], T.vp[f][r] = c[r];
      }
      f32x4_t s[MQ][2] = {};
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const uint32_t w = T.k[f][j], w8 = w >> 8;
          const u32x4_t a = {w & 0x000F000Fu, w & 0x00F000F0u, w8 & 0x000F000Fu, w8 & 0x00F000F0u};
#pragma unroll
          for (int i = 0; i < MQ; ++i) s[i][f] = mfma16(a, qf[i][j], s[i][f]);
        }
      __builtin_amdgcn_sched_barrier(0);  // (else all codes are spread ahead, and registers spill)
      // does row i see this lane's token 16 f + 4 g4 + r
      auto seen = [&](int i, int f, int r) {
        const int t = t0 + 16 * f + 4 * g4 + r;
        return !CUT || (t < end_t && t < see[i] && !(off >> f & 1));
      };
      auto value_scale = [&](int f, int r) { return __uint_as_float(T.vp[f][r] & 0xFFFF0000u); };
      float svm[MQ], top[MQ];
#pragma unroll
      for (int i = 0; i < MQ; ++i) svm[i] = 0.f, top[i] = -INFINITY;
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float ks = __uint_as_float(T.kp[f][r] & 0xFFFF0000u), kz = float(T.kp[f][r] & 0xFFu);
#pragma unroll
          for (int i = 0; i < MQ; ++i) {
            float v = fmaf(fmaf(-kz, qsum[i], s[i][f][r]), ks * qs[i], -ref[i]);
            if (!seen(i, f, r)) v = -INFINITY;
            s[i][f][r] = v;
            top[i] = fmaxf(top[i], v);
            svm[i] = fmaxf(svm[i], seen(i, f, r) ? value_scale(f, r) : 0.f);
          }
        }
      bool up = false;
#pragma unroll
      for (int i = 0; i < MQ; ++i) up |= top[i] > above[i] || svm[i] > 128.f * sigma[i];
      if (__any(up)) {  // new references
#pragma unroll
        for (int i = 0; i < MQ; ++i) {
          float sn = fmaxf(svm[i], __shfl_xor(svm[i], 16));
          sn = fmaxf(fmaxf(sn, __shfl_xor(sn, 32)), sigma[i]);
          const float fs = sn > 0.f ? sigma[i] / sn : 0.f;
          sigma[i] = sn;
          sinv[i] = sn > 0.f ? 1.f / sn : 0.f;
          float t = fmaxf(top[i], __shfl_xor(top[i], 16));
          t = fmaxf(t, __shfl_xor(t, 32));
          const float mn = fmaxf(m[i], ref[i] + t), fm = exp2f(m[i] - mn), fo = fm * fs;
          if (mn > NONE) {
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
              for (int r = 0; r < 4; ++r) s[i][f][r] += ref[i] - mn;
            ref[i] = mn, above[i] = 7.f;
          }
          m[i] = mn;
          l[i] *= fm, zs[i] *= fo;
          float fr[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) fr[r] = __shfl(fo, 4 * g4 + r);
#pragma unroll
          for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][d][r] *= fr[r];
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const u32x4_t w = *reinterpret_cast<const u32x4_t*>(tile + f * HALF + AT_V + 4 * lane);
#pragma unroll
        for (int r = 0; r < 4; ++r) T.v[f][r] = w[r];
      }
      u32x4_t pf[MQ];
#pragma unroll
      for (int f = 0; f < 2; ++f)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          const float v0 = value_scale(f, r), v1 = value_scale(f, r + 1);
          const float z0 = float(T.vp[f][r] & 0xFFu), z1 = float(T.vp[f][r + 1] & 0xFFu);
#pragma unroll
          for (int i = 0; i < MQ; ++i) {
            const float p0 = __builtin_amdgcn_exp2f(s[i][f][r]);
            const float p1 = __builtin_amdgcn_exp2f(s[i][f][r + 1]);
            l[i] += p0 + p1;
            float w0 = p0 * (v0 * sinv[i]), w1 = p1 * (v1 * sinv[i]);
            if (CUT) {  // a hidden token's value may read as NaN, or be far above sigma
              if (s[i][f][r] == -INFINITY) w0 = 0.f;
              if (s[i][f][r + 1] == -INFINITY) w1 = 0.f;
            }
            // (the zeros take the rounded weights too: their errors go with c - z then, not with c)
            const f16x2_t w = __builtin_convertvector(f32x2_t{w0, w1}, f16x2_t);
            zs[i] = fmaf(float(w[0]), z0, zs[i]);
            zs[i] = fmaf(float(w[1]), z1, zs[i]);
            pf[i][2 * f + (r >> 1)] = __builtin_bit_cast(uint32_t, w);
          }
        }
      __builtin_amdgcn_sched_barrier(0);
      // value codes: channel 8 n + d, pairs of tokens
      if constexpr (DIM == 128) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {  // low and high halves of the words: channels 0-3 and 4-7
          u32x4_t w, w8;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            w[k] = __builtin_amdgcn_perm(T.v[k >> 1][2 * (k & 1) + 1], T.v[k >> 1][2 * (k & 1)],
                                         x ? 0x07060302u : 0x05040100u);
            w8[k] = w[k] >> 8;
          }
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const u32x4_t bv = (d & 2 ? w8 : w) & (d & 1 ? 0x00F000F0u : 0x000F000Fu);
#pragma unroll
            for (int i = 0; i < MQ; ++i) acc[i][4 * x + d] = mfma16(pf[i], bv, acc[i][4 * x + d]);
          }
        }
      } else {  // lanes n and n + 8 share a word: channels 0-3 and 4-7 of it
        const uint32_t sel = n < 8 ? 0x05040100u : 0x07060302u;
        u32x4_t w, w8;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          w[k] = __builtin_amdgcn_perm(T.v[k >> 1][2 * (k & 1) + 1], T.v[k >> 1][2 * (k & 1)], sel);
          w8[k] = w[k] >> 8;
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const u32x4_t bv = (d & 2 ? w8 : w) & (d & 1 ? 0x00F000F0u : 0x000F000Fu);
#pragma unroll
          for (int i = 0; i < MQ; ++i) acc[i][d] = mfma16(pf[i], bv, acc[i][d]);
        }
      }
    };

    // this wave's tiles
    if (count > 0) {
      for (int k = 0; k < DEPTH - 1; ++k) load(k);
      auto next = [&](int k, auto cut_c) {
        const unsigned off = bad >> (2 * (k & (DEPTH - 1))) & 3;
        load(k + DEPTH - 1);  // (to the place of the tile before this one, which has been read)
        wait_vm<(DEPTH - 1) * LOADS>();
        __builtin_amdgcn_sched_barrier(0);
        work(k, first + STEP * k, off, cut_c);
      };
      // whole tiles first, the rest (all of it from a page on that does not exist) in a loop of its own:
      // two bodies in one loop hold their sums in different registers, and copy them
      const int whole = end_t < see0 ? end_t : see0;
      int k = 0;
      for (; k < count && first + STEP * k + 32 <= whole && !(bad >> (2 * (k & (DEPTH - 1))) & 3); ++k)
        next(k, std::false_type{});
      for (; k < count; ++k) next(k, std::true_type{});
      wait_vm<0>();  // (loads past the end)
    }
#pragma unroll
    for (int i = 0; i < MQ; ++i) {
      l[i] += __shfl_xor(l[i], 16);
      l[i] += __shfl_xor(l[i], 32);
      zs[i] += __shfl_xor(zs[i], 16);
      zs[i] += __shfl_xor(zs[i], 32);
    }
    // channel of block d of this lane
    const int chunk16 = chunk_of(n);
    auto channel = [&](int d) {
      return DIM == 128 ? 8 * chunk16 + d : 8 * (chunk16 & 7) + 4 * (n >> 3) + d;
    };

    if constexpr (BY_ROWS) {
      constexpr int RR = 8 / ND;  // rows at a time: eight registers for the stages between lanes
      const bool alone = A.splits == 1;
      const float norm = DIM == 128 ? 0.08838834764831845f : 0.125f;
      const float sign = (__popc(unsigned(chunk16)) & 1) ? -norm : norm;
#pragma unroll
      for (int i = 0; i < MQ; ++i)
#pragma unroll
        for (int r0 = 0; r0 < 4; r0 += RR) {
          float o[8], mm[RR], sum[RR];
#pragma unroll
          for (int u = 0; u < RR; ++u) {
            const int r = r0 + u;
            const float z = __shfl(zs[i], 4 * g4 + r);
            sum[u] = __shfl(l[i], 4 * g4 + r), mm[u] = __shfl(m[i], 4 * g4 + r);
            // (a row that sees nothing: zeros)
            const float sg = __shfl(sigma[i], 4 * g4 + r);
            const float f = !alone ? sg : sum[u] == 0.f ? 0.f : sg / sum[u];
            float x[ND];
#pragma unroll
            for (int d = 0; d < ND; ++d) x[d] = f * (acc[i][d][r] * (d & 1 ? 0x1p20f : 0x1p24f) - z);
            if (alone && A.rotate) hadamard_reg<ND>(x);
#pragma unroll
            for (int d = 0; d < ND; ++d) o[ND * u + d] = x[d];
          }
          if (alone && A.rotate) {
            stage_lane1(o, (chunk16 & 1) ? -1.f : 1.f);
            stage_lane2(o, (chunk16 & 2) ? -1.f : 1.f);
            stage_mirror8(o, (chunk16 & 4) ? -1.f : 1.f);
            stage_lane8(o, (chunk16 & 8) ? -1.f : 1.f);
#pragma unroll
            for (int d = 0; d < 8; ++d) o[d] *= sign;
          }
#pragma unroll
          for (int u = 0; u < RR; ++u) {
            const int row = row0 + 16 * i + 4 * g4 + r0 + u;
            if (row >= nrows) continue;
            const int64_t tok = q0 + row / G;
            const int head = h * G + row % G;
            const float* const x = o + ND * u;
            if (!alone) {
              const int64_t at = (int64_t(split) * A.n_tokens + tok) * A.n_heads + head;
#pragma unroll
              for (int d = 0; d < ND; d += 4)
                *reinterpret_cast<f32x4_t*>(A.part + at * DIM + channel(d)) =
                    f32x4_t{x[d], x[d + 1], x[d + 2], x[d + 3]};
              if (n == 0) A.ml[2 * at] = mm[u], A.ml[2 * at + 1] = sum[u];
              continue;
            }
            uint16_t* const out = A.out + tok * A.ldo + int64_t(head) * DIM + channel(0);
            if (A.wide) {
              uint32_t w[ND / 2];
#pragma unroll
              for (int d = 0; d < ND; d += 2)
                w[d / 2] = uint32_t(f32_bf16(x[d])) | uint32_t(f32_bf16(x[d + 1])) << 16;
              if constexpr (ND == 8)
                *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
              else
                *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
            } else {
#pragma unroll
              for (int d = 0; d < ND; ++d) out[d] = f32_bf16(x[d]);
            }
          }
        }
      continue;
    }
    // the waves' parts to LDS, where their tiles were
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MQ; ++i) {
      float* o = sm + (wave * ROWS + 16 * i) * LD;
      if (g4 == 0) {
        sml[(wave * ROWS + 16 * i + n) * 2] = m[i];
        sml[(wave * ROWS + 16 * i + n) * 2 + 1] = l[i];
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float z = __shfl(zs[i], 4 * g4 + r), sg = __shfl(sigma[i], 4 * g4 + r);
#pragma unroll
        for (int d = 0; d < ND; ++d)
          o[(4 * g4 + r) * LD + channel(d)] =
              sg * (acc[i][d][r] * (d & 1 ? 0x1p20f : 0x1p24f) - z);
      }
    }
    __syncthreads();
    for (int row = wave; row < end_row - row0; row += 4) {
      float mm[4], mx = -INFINITY, sum = 0.f, x[2] = {};
#pragma unroll
      for (int w = 0; w < 4; ++w) mm[w] = sml[(w * ROWS + row) * 2], mx = fmaxf(mx, mm[w]);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = exp2f(mm[w] - mx);
        sum += f * sml[(w * ROWS + row) * 2 + 1];
        x[0] += f * sm[(w * ROWS + row) * LD + lane];
        if constexpr (DIM == 128) x[1] += f * sm[(w * ROWS + row) * LD + lane + 64];
      }
      const int64_t tok = q0 + (row0 + row) / G;
      const int head = h * G + (row0 + row) % G;
      if (A.splits > 1) {
        const int64_t at = (int64_t(split) * A.n_tokens + tok) * A.n_heads + head;
        A.part[at * DIM + lane] = x[0];
        if constexpr (DIM == 128) A.part[at * DIM + lane + 64] = x[1];
        if (lane == 0) A.ml[2 * at] = mx, A.ml[2 * at + 1] = sum;
      } else {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;  // a row that sees nothing: zeros
        x[0] *= inv, x[1] *= inv;
        store_row<DIM>(A.out + tok * A.ldo + int64_t(head) * DIM, x, lane, A.rotate);
      }
    }
    __syncthreads();
  }
}

// the splits of a row (a wave each)
template <int DIM>
__global__ __launch_bounds__(256) void attention_join(AttnArgs A, int n_seqs) {
  const int lane = threadIdx.x & 63;
  const int64_t row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6), rows = A.n_tokens * A.n_heads;
  if (row >= rows) return;
  const int64_t tok = row / A.n_heads;
  if (A.starts) {  // tokens of no sequence were not computed
    bool in = false;
    for (int b = lane; b < n_seqs; b += 64) in |= tok >= A.starts[b] && tok < A.starts[b + 1];
    if (!__any(in)) return;
  }
  float mx = -INFINITY;
  for (int s = 0; s < A.splits; ++s) mx = fmaxf(mx, A.ml[2 * (s * rows + row)]);
  float x[2] = {}, sum = 0.f;
  for (int s = 0; s < A.splits; ++s) {
    const int64_t at = s * rows + row;
    const float f = exp2f(A.ml[2 * at] - mx);
    sum += f * A.ml[2 * at + 1];
    x[0] += f * A.part[at * DIM + lane];
    if constexpr (DIM == 128) x[1] += f * A.part[at * DIM + lane + 64];
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  x[0] *= inv, x[1] *= inv;
  store_row<DIM>(A.out + tok * A.ldo + (row % A.n_heads) * DIM, x, lane, A.rotate);
}

// zeros for tokens of no sequence where there is no sequence at all
__global__ __launch_bounds__(256) void cache_zeros(uint16_t* out, int64_t ldo, int64_t n_tokens,
                                                   int width) {
  for (int64_t t = blockIdx.x; t < n_tokens; t += gridDim.x)
    for (int e = threadIdx.x; e < width; e += 256) out[t * ldo + e] = 0;
}

// ---- plan and launches ---------------------------------------------------------------------------
constexpr int64_t MAX_SPLITS = 32, SPLIT_ROWS = 131072;

// rows of partial outputs that the workspace holds
int64_t split_rows(int64_t rows) {
  return rows * MAX_SPLITS < SPLIT_ROWS + rows ? rows * MAX_SPLITS : SPLIT_ROWS + rows;
}

template <int DIM, int MQ, bool BY_ROWS>
int launch_attention(const AttnArgs& a, int64_t n_seqs, hipStream_t s) {
  const size_t tiles = size_t(4) * DEPTH * tile_words(DIM) * 4;
  const size_t ends = BY_ROWS ? 0 : size_t(4) * 16 * MQ * (DIM + 4 + 2) * sizeof(float);
  const size_t lds = tiles > ends ? tiles : ends;
  const dim3 grid(static_cast<unsigned>(a.n_kv), static_cast<unsigned>(n_seqs),
                  static_cast<unsigned>(a.tiles * a.splits));
  KQ_TRY(launch("cache_attention", cache_attention<DIM, MQ, BY_ROWS>, grid, dim3(256), lds, s, a));
  if (a.splits == 1) return KRONQ_OK;
  return launch("attention_join", attention_join<DIM>,
                dim3(static_cast<unsigned>(cdiv(a.n_tokens * a.n_heads, 4))), dim3(256), 0, s, a,
                int(n_seqs));
}

}  // namespace

int cache_append_launch(const AppendJob& j, hipStream_t s) {
  AppendArgs a{};
  a.k = j.k, a.v = j.v, a.ldk = j.ldk, a.ldv = j.ldv, a.n_tokens = j.n_tokens;
  a.n_kv = int(j.n_kv), a.page_log = __builtin_ctzll(uint64_t(j.page));
  a.n_slots = j.n_pages * j.page, a.slots = j.slots, a.codes = j.codes, a.params = j.params;
  a.rotate = j.rotate, a.norm = 1.0 / std::sqrt(double(j.dim)), a.k_hat = j.k_hat, a.v_hat = j.v_hat;
  const dim3 grid = grid_of(cdiv(j.n_tokens * j.n_kv * 2, 2048 / j.dim));
  const bool half = j.dtype == KRONQ_BF16;
  if (j.dim == 128)
    return half ? launch("cache_append", cache_append<uint16_t, 128>, grid, dim3(256), 0, s, a)
                : launch("cache_append", cache_append<float, 128>, grid, dim3(256), 0, s, a);
  return half ? launch("cache_append", cache_append<uint16_t, 64>, grid, dim3(256), 0, s, a)
              : launch("cache_append", cache_append<float, 64>, grid, dim3(256), 0, s, a);
}

size_t attention_ws_bytes(int64_t n_heads, int64_t dim, int64_t n_tokens) {
  if (n_heads <= 0 || dim <= 0 || n_tokens <= 0) return 0;
  const size_t rows = size_t(split_rows(n_heads * n_tokens));
  return align256(rows * size_t(dim) * 4) + align256(rows * 8);
}

int cache_zeros_launch(void* out, int64_t ldo, int64_t n_tokens, int64_t width, hipStream_t s) {
  const int64_t groups = n_tokens < 65536 ? n_tokens : 65536;
  return launch("cache_zeros", cache_zeros, dim3(static_cast<unsigned>(groups)), dim3(256), 0, s,
                static_cast<uint16_t*>(out), ldo, n_tokens, int(width));
}

int cache_attention_launch(const AttentionJob& j, void* ws, hipStream_t s) {
  AttnArgs a{};
  a.q = static_cast<const uint16_t*>(j.q), a.ldq = j.ldq, a.n_tokens = j.n_tokens;
  a.n_heads = int(j.n_heads), a.n_kv = int(j.n_kv), a.group = int(j.n_heads / j.n_kv);
  a.codes = j.codes, a.params = j.params, a.n_pages = j.n_pages;
  a.page_log = __builtin_ctzll(uint64_t(j.page));
  a.table = j.table, a.ldt = j.ldt, a.table_pages = int(j.table_pages), a.lengths = j.lengths;
  a.starts = j.starts, a.scale = j.scale * 1.4426950408889634f;
  a.rotate = (j.flags & KRONQ_CACHE_ROTATE) != 0, a.fill = (j.flags & KRONQ_CACHE_FILL) != 0;
  a.out = static_cast<uint16_t*>(j.out), a.ldo = j.ldo;
  a.wide = aligned(j.out, 16) && j.ldo % 8 == 0;
  // Up to 64 rows of a sequence and kv head share their tokens out to the waves (two tiles of 32 rows
  // from 33 on); more are walked by 128 rows a workgroup, which read the tokens once for all of them.
  const int64_t rows = j.max_new * a.group;
  const bool by_rows = rows > 64;
  const int mq = rows <= 16 ? 1 : 2;
  a.tiles = int(cdiv(rows, by_rows ? 64 * mq : 16 * mq));
  // Enough workgroups for sequences of different lengths to even out, of 256 tokens each at least (48
  // decoding sequences of up to 16384 tokens: 130 us with 1024 of them, 129 with 1536, 135 with 2048).
  // (without starts, sequences from n_tokens on have no new token)
  const int64_t n_seqs = j.starts || j.n_seqs < j.n_tokens ? j.n_seqs : j.n_tokens;
  const int64_t wgs = a.tiles * j.n_kv * n_seqs, all = j.n_tokens * j.n_heads;
  int64_t splits = cdiv(by_rows ? 512 : 1536, wgs);
  // (decoding over up to 512 tokens goes undivided: the second launch costs a call 3 of 17 us, and
  // two tiles of a wave less gain about as much on the device as joining takes)
  const int64_t room = j.table_pages * j.page;
  const int64_t useful = !by_rows && room <= 512 ? 1 : cdiv(room, 256);
  splits = splits < useful ? splits : useful;
  splits = splits < MAX_SPLITS ? splits : MAX_SPLITS;
  if (splits * all > split_rows(all)) splits = split_rows(all) / all;
  a.splits = int(splits < 1 ? 1 : splits);
  // (the last dimension of the grid: more tiles are walked in turn)
  a.tiles = a.tiles * a.splits <= 65535 ? a.tiles : 65535 / a.splits;
  Carver cv(ws);
  const size_t cap = size_t(split_rows(all));
  a.part = cv.take<float>(cap * size_t(j.dim));
  a.ml = cv.take<float>(cap * 2);
  if (j.dim == 128)
    return mq == 1   ? launch_attention<128, 1, false>(a, n_seqs, s)
           : by_rows ? launch_attention<128, 2, true>(a, n_seqs, s)
                     : launch_attention<128, 2, false>(a, n_seqs, s);
  return mq == 1   ? launch_attention<64, 1, false>(a, n_seqs, s)
         : by_rows ? launch_attention<64, 2, true>(a, n_seqs, s)
                   : launch_attention<64, 2, false>(a, n_seqs, s);
}

}  // namespace kq
