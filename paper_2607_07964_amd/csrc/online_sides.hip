// Both sides of the served layer (online_linear.hip): the transform of the activations to fp16 in
// fragment order, and the transform of the products with bias, activation and residual.
//
// A transform of order d is A (x) H_m with A = Q28 (or its transpose), or H_d alone. A workgroup of
// 256 threads takes a row, as d / cols columns of cols = min(m, 512) elements. Its two factors touch
// the row in two ways that meet once in LDS:
//   across the columns (A and the upper stages of H): a thread holds the same two elements of every
//     column, 2 d / cols registers, and mixes them in place (A = Q28: mix28);
//   inside a column (the lower nine stages of H): a lane holds 8 neighbours, three stages in
//     registers, six across lanes by DPP.
// The input side goes across first, straight from the row in memory, and ends with 8 neighbours per
// lane, which is what a 16-byte piece in fragment order takes; the output side goes the other way
// round, and its epilogue works on neighbours of neighbouring threads. Bound by the reads and writes
// of the rows; with a 28-point factor by its 28 multiply-adds per element.
#include <cmath>

#include "kq_fwht.hpp"
#include "kq_linear.hpp"

namespace kq {
namespace {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_f32(uint32_t h) { return __uint_as_float(h << 16); }
// rounded to nearest even; NaN stays NaN
__device__ __forceinline__ uint16_t f32_bf16(float v) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float(uint32_t(127 + e) << 23); }
__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// The expert whose rows [offsets[e], offsets[e + 1]) hold this one, or -1. Every thread of the
// workgroup calls it.
__device__ __forceinline__ int expert_of(const int* offsets, int n_experts, int64_t row) {
  int n = 0;  // experts whose range ends at or before the row
  for (int e0 = 0; e0 < n_experts; e0 += int(blockDim.x)) {
    const int e = e0 + int(threadIdx.x);
    n += __syncthreads_count(e < n_experts && offsets[e + 1] <= row);
  }
  return n >= n_experts || row < offsets[0] ? -1 : n;
}

// The list of tiles, by one workgroup: the experts' ranges made ascending and cut to
// [0, n_rows), so that no content of offsets leads out of the rows.
__device__ void list_tiles(const LinearIn& A, int* sh) {
  const int tid = threadIdx.x, thr = blockDim.x, n = int(A.n_rows);
  int base = 0, top = clampi(A.offsets[0], 0, n);  // tiles so far, largest offset so far
  for (int e0 = 0; e0 < A.n_experts; e0 += thr) {
    const int e = e0 + tid;
    int v = e < A.n_experts ? clampi(A.offsets[e + 1], 0, n) : 0;
    for (int o = 1; o < thr; o <<= 1) {  // running maximum over the threads
      sh[tid] = v;
      __syncthreads();
      if (tid >= o) v = max(v, sh[tid - o]);
      __syncthreads();
    }
    v = max(v, top);
    sh[tid] = v;
    __syncthreads();
    const int lo = tid ? sh[tid - 1] : top, hi = v;
    top = sh[thr - 1];
    __syncthreads();
    const int u0 = lo >> 5, nu = hi > lo ? ((hi - 1) >> 5) - u0 + 1 : 0;
    const int k = (nu + A.nt - 1) / A.nt;
    int sum = k;  // (running over the threads)
    for (int o = 1; o < thr; o <<= 1) {
      sh[tid] = sum;
      __syncthreads();
      if (tid >= o) sum += sh[tid - o];
      __syncthreads();
    }
    if (e < A.n_experts) A.first[e] = make_int2(base + sum - k, u0);
    for (int i = 0; i < k; ++i) {
      const int64_t at = base + sum - k + i;
      if (at < A.max_tiles) A.tiles[1 + at] = LinearTile{e, u0 + i * A.nt, lo, hi};
    }
    sh[tid] = sum;
    __syncthreads();
    base += sh[thr - 1];
    __syncthreads();
  }
  if (tid == 0) A.tiles[0] = LinearTile{base < A.max_tiles ? base : int(A.max_tiles), 0, 0, 0};
}

// The table of a workgroup's TABLE_ROWS rows of W, 32 groups at a time, turned in LDS (sh): the rows
// are read along their groups and the table is written along its rows, in whole lines.
constexpr int TABLE_ROWS = 32, TABLE_LDS = 32 * (TABLE_ROWS + 1);
template <int THR>
__device__ void fill_table(const LinearIn& A, int64_t block, int* sh) {
  constexpr int PER = THR / TABLE_ROWS;  // threads of a row
  const int r = threadIdx.x / PER, t = threadIdx.x % PER;
  const int64_t row0 = block * TABLE_ROWS, row = row0 + r < A.w_rows ? row0 + r : A.w_rows - 1;
  const float *s = A.scales + row * A.ldsz, *z = A.zeros + row * A.ldsz;
  const int nq = A.ng / A.gpq;
  float mx = 0.f;
  for (int g = t; g < nq; g += PER) mx = fmaxf(mx, fabsf(s[g]));
#pragma unroll
  for (int o = 1; o < PER; o <<= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
  // the largest s / unit in [2^4, 2^5): |s (c - z)| / unit < 2^5 * 1280, inside fp16, and groups down to
  // 2^-14 of the row's largest scale stay normal beside the shifted codes (times 2^-4)
  const int e = int(__float_as_uint(mx) >> 23) - 127;
  const int ue = mx > 0.f && e < 128 ? clampi(e - 4, -122, 123) : 0;
  const float up = pow2f(-ue);
  if (t == 0) A.w_unit[row] = pow2f(ue);
  for (int g0 = 0; g0 < A.ng; g0 += 32) {
    for (int g = g0 + t; g < g0 + 32 && g < A.ng; g += PER) {
      const int q = g / A.gpq;
      const f16x2_t o = {_Float16(s[q] * up), _Float16(-1024.f - z[q])};
      sh[(g - g0) * (TABLE_ROWS + 1) + r] = __builtin_bit_cast(int, o);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * TABLE_ROWS; i += THR) {
      const int g = i / TABLE_ROWS, to = i % TABLE_ROWS;
      if (g0 + g < A.ng && row0 + to < A.w_rows)
        A.table[int64_t(g0 + g) * A.w_rows + row0 + to] = uint32_t(sh[g * (TABLE_ROWS + 1) + to]);
    }
    __syncthreads();
  }
}

// The octet of a wave's 64 that a lane holds: lanes 4-7 of each 8 in reverse order, so that the
// octet 4 further on is the mirrored lane of the 8 (one DPP control) and not two exchanges away.
__device__ __forceinline__ int octet_of(int lane) { return lane ^ ((lane & 4) ? 3 : 0); }
// Strides 8 ... 64 are single multiply-adds with the partner read by DPP (kq_fwht.hpp), which leave
// each value times this sign of its octet: the callers multiply by it once.
__device__ __forceinline__ float octet_sign(int octet, int cols) {
  return (__popc(unsigned(octet & 15 & (cols / 8 - 1))) & 1) ? -1.f : 1.f;
}

// (every lane of the wave comes here; FULL: columns of 512)
template <int N, bool FULL>
__device__ __forceinline__ void stages_dpp(float (&x)[8 * N], int octet, int cols) {
  const float s0 = (octet & 1) ? -1.f : 1.f, s1 = (octet & 2) ? -1.f : 1.f;
  const float s2 = (octet & 4) ? -1.f : 1.f, s3 = (octet & 8) ? -1.f : 1.f;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    float* v = x + 8 * n;
    if (FULL || cols >= 128) {
      stage_lane1(v, s0);
      stage_lane2(v, s1);
      stage_mirror8(v, s2);
      stage_lane8(v, s3);
    } else {
      if (cols > 8) stage_lane1(v, s0);
      if (cols > 16) stage_lane2(v, s1);
      if (cols > 32) stage_mirror8(v, s2);
    }
  }
}

// registers k and k + 4 of each octet: sum and difference
template <int N>
__device__ __forceinline__ void stage_high(float (&x)[8 * N]) {
#pragma unroll
  for (int e = 0; e < 8 * N; ++e)
    if (!(e & 4)) {
      const float a = x[e], b = x[e + 4];
      x[e] = a + b, x[e + 4] = a - b;
    }
}
// exchange registers k + 4 of the lower 16 lanes (of each 32) or 32 lanes with registers k of the
// upper: bit 2 of the register takes the place of lane bit 4 or 5, and that bit its place
template <int N, bool WIDE>
__device__ __forceinline__ void turn_high(float (&x)[8 * N]) {
#pragma unroll
  for (int e = 0; e < 8 * N; ++e)
    if (!(e & 4)) {
      const uint32_t a = __float_as_uint(x[e]), b = __float_as_uint(x[e + 4]);
      if constexpr (WIDE) {
        const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
        x[e] = __uint_as_float(r[0]), x[e + 4] = __uint_as_float(r[1]);
      } else {
        const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
        x[e] = __uint_as_float(r[0]), x[e + 4] = __uint_as_float(r[1]);
      }
    }
}

// The stages inside a column on octets of neighbours (octet_of the lane in each of N), up to
// octet_sign. Elements 2^2, 2^7 and 2^8 apart are brought into one register bit, one after another.
// What a lane holds at the start and at the end differs with columns of 512: register bit 2 and lane
// bits 4 and 5 stand for element bits
//   8-neighbours first:  (2, 7, 8) at the start, (8, 2, 7) at the end;
//   8-neighbours last:   (7, 8, 2) at the start, (2, 7, 8) at the end.
template <int N, bool FULL>
__device__ __forceinline__ void inside_column(float (&x)[8 * N], int lane, int cols) {
#pragma unroll
  for (int e = 0; e < 8 * N; e += 4) {
    float v[4] = {x[e], x[e + 1], x[e + 2], x[e + 3]};
    hadamard_reg<4>(v);
    x[e] = v[0], x[e + 1] = v[1], x[e + 2] = v[2], x[e + 3] = v[3];
  }
  stages_dpp<N, FULL>(x, octet_of(lane), cols);
  stage_high<N>(x);
  if (!FULL && cols < 256) return;
  turn_high<N, false>(x);
  stage_high<N>(x);
  if constexpr (FULL) {
    turn_high<N, true>(x);
    stage_high<N>(x);
  } else {
    turn_high<N, false>(x);  // (back)
  }
}
// first element of registers 4 h to 4 h + 3 of a lane before (first) or after inside_column, among
// the 512 of a wave
template <bool FIRST, bool FULL>
__device__ __forceinline__ int quad_at(int lane, int h) {
  const int o = octet_of(lane), b4 = (lane >> 4) & 1, b5 = lane >> 5;
  if (!FULL) return 8 * o + 4 * h;
  return FIRST ? 8 * ((o & 15) | h << 4 | b4 << 5) + 4 * b5
               : 8 * ((o & 15) | b5 << 4 | h << 5) + 4 * b4;
}

// H_C over the columns of two elements: put(c, x, y) takes the results.
template <int C, typename Put>
__device__ __forceinline__ void across_columns(float (&x)[C], float (&y)[C], Put put) {
  hadamard_reg<C>(x);
  hadamard_reg<C>(y);
#pragma unroll
  for (int c = 0; c < C; ++c) put(c, x[c], y[c]);
}

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// The factor in LDS (its rows 28 floats apart; as loads of every lane's own values it was a third of
// the time of linear_in), and a lane's share of it, or of its transpose, as the A operand of mix28
template <int THR>
__device__ __forceinline__ void stage28(float* lds, const float* __restrict__ q28, int tid) {
  for (int i = tid; i < 784; i += THR) lds[i] = q28[i];
}
template <bool TRANS>
__device__ __forceinline__ void load28(float (&q)[14], const float* lds, int lane) {
#pragma unroll
  for (int s = 0; s < 14; ++s) {
    const int k = 2 * s + (lane >> 5), n = lane & 31, a = n < 28 ? n : 27;
    q[s] = lds[TRANS ? k * 28 + a : a * 28 + k];  // (rows 28 to 31 are not used)
  }
}

// The 28 x 28 factor over the segments of m elements of the row in LDS, on the fp32 matrix cores (as
// multiply-adds of a thread's own elements it took three times as long: two chains of 28 at a time),
// and, for m = 1024 (B = 2), the stage of stride 512 that a column of 512 leaves out. A wave takes
// 32 places of every segment at a time; place(i, v): element i of the row has become v.
template <int B, typename Place>
__device__ __forceinline__ void mix28(const float* buf, int m, const float (&q)[14], int wave,
                                      int waves, int lane, Place place) {
  const int n = lane & 31, half = lane >> 5;
  const int cols = B == 2 ? 512 : m;
  for (int p0 = 32 * wave; p0 < cols; p0 += 32 * waves) {
    const int p = p0 + n, pc = p < cols ? p : cols - 1;
    f32x16_t d[B] = {};
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
      for (int s = 0; s < 14; ++s)
        d[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(q[s], buf[(2 * s + half) * m + 512 * b + pc],
                                                    d[b], 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int a = 8 * (r >> 2) + 4 * half + (r & 3);
      if (a >= 28 || p >= cols) continue;
      if constexpr (B == 2) {
        place(a * m + p, d[0][r] + d[1][r]);
        place(a * m + p + 512, d[0][r] - d[1][r]);
      } else {
        place(a * m + p, d[0][r]);
      }
    }
  }
}

__device__ __forceinline__ void load2(const uint16_t* p, float& a, float& b) {
  const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
  a = __uint_as_float(w << 16), b = __uint_as_float(w & 0xFFFF0000u);
}
__device__ __forceinline__ void load2(const float* p, float& a, float& b) {
  const float2 w = *reinterpret_cast<const float2*>(p);
  a = w.x, b = w.y;
}
__device__ __forceinline__ void load8(const uint16_t* p, float* v) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int k = 0; k < 4; ++k)
    v[2 * k] = __uint_as_float(u[k] << 16), v[2 * k + 1] = __uint_as_float(u[k] & 0xFFFF0000u);
}
__device__ __forceinline__ void load8(const float* p, float* v) {
#pragma unroll
  for (int k = 0; k < 8; k += 4) {
    const float4 w = *reinterpret_cast<const float4*>(p + k);
    v[k] = w.x, v[k + 1] = w.y, v[k + 2] = w.z, v[k + 3] = w.w;
  }
}

// Threads of a workgroup. A row of 28 m takes most of the LDS of half a CU: 16 waves hide its steps.
constexpr int threads(int c) { return c && c % 28 == 0 ? 1024 : 256; }
// (linear_in's short rows need no more, and have twice the workgroups on a CU)
constexpr int in_threads(int c) { return c == 1 || c == 2 ? 128 : threads(c); }

// C: columns of a rotated row (0: not rotated), of 512 elements with FULL. N: octets a thread ends with.
template <typename T, int C, int N, bool FULL>
__global__ __launch_bounds__(in_threads(C)) void linear_in(LinearIn A, int table_blocks, int lead) {
  extern __shared__ __attribute__((aligned(16))) float buf[];  // the row, when rotated
  constexpr int THR = in_threads(C), WAVES = THR / 64;
  __shared__ float red[WAVES];
  __shared__ int sh[TABLE_LDS];  // (also a workgroup's threads, or the factor)
  static_assert(TABLE_LDS >= THR && TABLE_LDS >= 784);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t group = workgroup();
  if (group < lead) {
    if (group < table_blocks) fill_table<THR>(A, group, sh);
    if (group == lead - 1 && A.offsets) list_tiles(A, sh);
    return;
  }
  // The rows of a unit on one XCD (group % 8; lead is a multiple of 8), one after another: a
  // line of the result holds 8 rows, and is then complete before it leaves that XCD's L2.
  const int64_t b = group - lead, in = b >> 3;
  const int64_t row = ((b & 7) + 8 * (in >> 5)) * 32 + (in & 31);
  if (row >= A.n_rows) return;
  int expert = 0;
  if (A.offsets) {
    expert = expert_of(A.offsets, A.n_experts, row);
    if (expert < 0) return;
  }
  const int d = int(A.d_in);
  const T* x = static_cast<const T*>(A.x) + row * A.ldx;
  const float* mul = A.mul ? A.mul + int64_t(expert) * d : nullptr;
  float v[8 * N];
  if constexpr (C > 0) {
    const int cols = A.turn.cols;
    if constexpr (C % 28 == 0) {
      float* const factor = reinterpret_cast<float*>(sh);
      stage28<THR>(factor, A.q28 + int64_t(expert) * 784, tid);
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int j = 8 * (tid + THR * n);
        if (j >= d) continue;
        float o[8];
        load8(x + j, o);
        if (mul) {
          float f[8];
          load8(mul + j, f);
#pragma unroll
          for (int k = 0; k < 8; ++k) o[k] *= f[k];
        }
        *reinterpret_cast<float4*>(buf + j) = make_float4(o[0], o[1], o[2], o[3]);
        *reinterpret_cast<float4*>(buf + j + 4) = make_float4(o[4], o[5], o[6], o[7]);
      }
      __syncthreads();
      float q[14];
      load28<false>(q, factor, lane);
      // (in place: a wave reads all of its 32 places before it writes them)
      mix28<C / 28>(buf, A.turn.m, q, wave, WAVES, lane, [&](int i, float v) { buf[i] = v; });
    } else {
      for (unsigned p = 2 * tid; int(p) < cols; p += 2 * THR) {
        float u[C], w[C];
#pragma unroll
        for (int c = 0; c < C; ++c) load2(x + c * cols + p, u[c], w[c]);
        if (mul) {
#pragma unroll
          for (int c = 0; c < C; ++c) {
            const float2 f = *reinterpret_cast<const float2*>(mul + c * cols + p);
            u[c] *= f.x, w[c] *= f.y;
          }
        }
        across_columns<C>(u, w, [&](int c, float a, float b) {
          *reinterpret_cast<float2*>(buf + c * cols + p) = make_float2(a, b);
        });
      }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int j = 512 * (wave + WAVES * n) + quad_at<true, FULL>(lane, h);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        if (j < d) o = *reinterpret_cast<const float4*>(buf + j);
        v[8 * n + 4 * h] = o.x, v[8 * n + 4 * h + 1] = o.y;
        v[8 * n + 4 * h + 2] = o.z, v[8 * n + 4 * h + 3] = o.w;
      }
    inside_column<N, FULL>(v, lane, cols);
  } else {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int j = 8 * (64 * (wave + WAVES * n) + octet_of(lane));
      float o[8] = {};
      if (j < d) {
        load8(x + j, o);
        if (mul) {
          float f[8];
          load8(mul + j, f);
#pragma unroll
          for (int k = 0; k < 8; ++k) o[k] *= f[k];
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) v[8 * n + k] = o[k];
    }
  }
  // the row's largest value to [2^7, 2^8)
  float mx = 0.f;
#pragma unroll
  for (int k = 0; k < 8 * N; ++k) mx = fmaxf(mx, fabsf(v[k]));
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
  if (lane == 0) red[wave] = mx;
  __syncthreads();
  mx = red[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) mx = fmaxf(mx, red[i]);
  mx *= A.turn.norm;
  const int e = int(__float_as_uint(mx) >> 23) - 127;
  // (up to fp32's largest; below 2^-112 the row is left smaller, and its unit a normal number)
  const int ue = mx > 0.f && e < 128 ? clampi(e - 7, -119, 120) : 0;
  float up = pow2f(-ue) * A.turn.norm;
  if (tid == 0) A.row_unit[row] = pow2f(ue);
  const int octet = octet_of(lane);
  if constexpr (C > 0) up *= octet_sign(octet, A.turn.cols);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int j = 8 * (64 * (wave + WAVES * n) + octet);
    float o[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      o[k] = v[8 * n + k] * up;
      asm("" : "+v"(o[k]));  // both planes from the one rounded product (a multiplication merged
    }                        // into one conversion only would round the planes' sum twice)
    // Octet oc of its chunk of 32 columns is step oc of the codes, its elements in the order in which a
    // packed chunk's codes are spread to pairs of fp16: columns k and k + 4 (3 and 4 bits), k and k + 2
    // of either half (8 bits); with 2 bits a step takes columns k and k + 8, four of either of two octets,
    // which lie in neighbouring lanes.
    float t[8];
    if (A.bits == 2) {
      const bool odd = octet & 1;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float got = dpp_mov<0xB1>(odd ? o[k] : o[4 + k]);
        t[2 * k] = odd ? got : o[k];
        t[2 * k + 1] = odd ? o[4 + k] : got;
      }
    } else if (A.bits == 8) {
      t[0] = o[0], t[1] = o[2], t[2] = o[1], t[3] = o[3];
      t[4] = o[4], t[5] = o[6], t[6] = o[5], t[7] = o[7];
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) t[2 * k] = o[k], t[2 * k + 1] = o[4 + k];
    }
    if (j >= d) continue;
    f16x8_t hi;
#pragma unroll
    for (int k = 0; k < 8; ++k) hi[k] = _Float16(t[k]);
    const int ks = (j >> 7) * 8 + ((j >> 5) & 1) * 4 + ((j >> 3) & 3), h = (j >> 6) & 1;
    uint16_t* to = A.xf + (((row >> 5) * (d / 16) + ks) * 64 + (row & 31) + 32 * h) * 8;
    *reinterpret_cast<f16x8_t*>(to) = hi;
    if (A.planes == 2) {
      f16x8_t lo;
#pragma unroll
      for (int k = 0; k < 8; ++k) lo[k] = _Float16(t[k] - float(hi[k]));
      *reinterpret_cast<f16x8_t*>(to + A.plane) = lo;
    }
  }
}

__device__ __forceinline__ float activate(float z, int act) {
  switch (act) {
    case KRONQ_ACT_RELU:
      return z < 0.f ? 0.f : z;  // (NaN stays)
    case KRONQ_ACT_GELU:
      return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    case KRONQ_ACT_SILU:
      return z / (1.f + expf(-z));
    default:
      return z;
  }
}

template <typename T>
__device__ __forceinline__ float load1(const void* p, int64_t i) {
  if constexpr (sizeof(T) == 2) return bf16_f32(static_cast<const uint16_t*>(p)[i]);
  return static_cast<const float*>(p)[i];
}

template <typename T>
__device__ __forceinline__ void store1(void* p, int64_t i, float v) {
  if constexpr (sizeof(T) == 2)
    static_cast<uint16_t*>(p)[i] = f32_bf16(v);
  else
    static_cast<float*>(p)[i] = v;
}

// multiplier, bias, activation and residual of element j of a row (mul, bias and residual are the
// row's, or null)
template <typename T>
__device__ __forceinline__ float finish(float v, unsigned j, const float* mul, const float* bias,
                                        const T* residual, int act) {
  if (mul) v *= mul[j];
  if (bias) v += bias[j];
  v = activate(v, act);
  if (residual) v += load1<T>(residual, j);
  return v;
}

// Where a row's products lie.
struct Products {
  const LinearOut& A;
  const float* p;
  const float* w_unit;
  int64_t row;
  int item0, in_tile, full_items, per;  // dealt

  __device__ __forceinline__ Products(const LinearOut& a, int64_t r, int expert) : A(a), row(r) {
    p = A.part + row * A.ld;
    w_unit = A.w_unit ? A.w_unit + int64_t(expert) * A.d_out : nullptr;
    if (A.workers == 0) return;
    const int u = int(row >> 5);
    int ti = u / A.nt, unit = ti * A.nt, items = A.items;
    if (A.first) {
      const int2 f = A.first[expert];
      const int k = (u - f.y) / A.nt;
      ti = f.x + k, unit = f.y + k * A.nt;
      items = A.tiles[0].expert * A.row_blocks;
    }
    const LinearDeal d = linear_deal(items, A.ng, A.workers);
    // (offsets that do not ascend give tiles that do not hold the row: kept within the buffers)
    item0 = clampi(ti, 0, items / A.row_blocks) * A.row_blocks;
    in_tile = clampi(int(row) - unit * 32, 0, 32 * A.nt - 1);
    full_items = d.full * A.workers, per = d.per;
  }
  // the workers after the first one that hold parts of element j's item: [from, to)
  __device__ __forceinline__ void parts(int j, int& from, int& to) const {
    const int r = item0 + int(unsigned(j) / unsigned(LINEAR_BLOCK)) - full_items;
    from = to = 0;
    if (r < 0) return;
    from = r * A.ng / per + 1, to = ((r + 1) * A.ng - 1) / per + 1;
    to = to < A.workers ? to : A.workers;
  }
  __device__ __forceinline__ const float* kept(int worker, int j) const {
    return A.kept + (int64_t(worker) * 32 * A.nt + in_tile) * LINEAR_BLOCK + (j & (LINEAR_BLOCK - 1));
  }
  // eight neighbours
  __device__ __forceinline__ void sum8(int j, float* v) const {
    load8(p + j, v);
    float w[8];
    if (A.workers == 0) return;
    int from, to;
    parts(j, from, to);
    for (; from < to; from += 4) {  // (four at a time: they come one after another otherwise)
      float u[4][8];
#pragma unroll
      for (int i = 0; i < 4; ++i) load8(kept(from + i < to ? from + i : to - 1, j), u[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += from + i < to ? u[i][k] : 0.f;
    }
    if (w_unit) {
      load8(w_unit + j, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] *= w[k];
    }
  }
  // elements j + k step below d, their parts four at a time and all of them together: one after another
  // they wait for memory as often as there are parts
  template <int K>
  __device__ __forceinline__ void sum_each(int j, int step, int d, float (&v)[K]) const {
    int from[K], to[K], most = 0, at[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      at[k] = j + k * step < d ? j + k * step : j;
      v[k] = p[at[k]];
      from[k] = to[k] = 0;
      if (A.workers) parts(at[k], from[k], to[k]);
      most = max(most, to[k] - from[k]);
    }
    for (int s = 0; s < most; s += 4) {
      float u[K][4];
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int w = from[k] + s + i;
          u[k][i] = to[k] > from[k] ? *kept(w < to[k] ? w : to[k] - 1, at[k]) : 0.f;
        }
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[k] += from[k] + s + i < to[k] ? u[k][i] : 0.f;
    }
    if (w_unit) {
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] *= w_unit[at[k]];
    }
  }
};

// The epilogue on the row in LDS, times unit and the sign that its octets are left with: the elements
// of places p and p + 1 of every column c from c0 on, c1 apart, of the count elements from first on
// that buf holds. A loop, and not unrolled: the
// activations' code is long, a row is over before it comes from memory once (46 us for rows of 14336
// with 56 copies of it, for 23 rows and more alike).
template <typename T>
__device__ __forceinline__ void finish_row(const LinearOut& A, const float* buf, int64_t row,
                                           int expert, float unit, int p, int c0, int c1, int first,
                                           int count) {
  const int d = int(A.d_out), cols = A.turn.cols;
  const float* const mul = A.mul ? A.mul + int64_t(expert) * d + first : nullptr;
  const float* const bias = A.bias ? A.bias + int64_t(expert) * d + first : nullptr;
  const T* const res =
      A.residual ? static_cast<const T*>(A.residual) + row * A.ldr + first : nullptr;
  T* const y = static_cast<T*>(A.y) + row * A.ldy + first;
  const float up = unit * octet_sign(p >> 3, cols);
#pragma unroll 1
  for (unsigned j = c0 * cols + p; int(j) < count; j += c1 * cols) {
    const float2 v = *reinterpret_cast<const float2*>(buf + j);
    float a = v.x * up, b = v.y * up, f, g;
    if (mul) load2(mul + j, f, g), a *= f, b *= g;
    if (A.pairs) {
      if (bias) load2(bias + j, f, g), a += f, b += g;
      a = activate(a, A.act), b = activate(b, A.act);
      if (res) load2(res + j, f, g), a += f, b += g;
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint32_t*>(y + j) = uint32_t(f32_bf16(a)) | uint32_t(f32_bf16(b)) << 16;
      else
        *reinterpret_cast<float2*>(y + j) = make_float2(a, b);
    } else {
      if (bias) a += bias[j], b += bias[j + 1];
      a = activate(a, A.act), b = activate(b, A.act);
      if (res) a += load1<T>(res, j), b += load1<T>(res, j + 1);
      store1<T>(y, j, a);
      store1<T>(y, j + 1, b);
    }
  }
}

// C columns of a rotated row of whole octets
template <typename T, int C, bool FULL>
__global__ __launch_bounds__(threads(C)) void linear_out(LinearOut A) {
  extern __shared__ __attribute__((aligned(16))) float buf[];  // the row
  constexpr int THR = threads(C), WAVES = THR / 64, N = (64 * C + THR - 1) / THR;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int d = int(A.d_out), cols = A.turn.cols;
  const int64_t row = workgroup();
  if (row >= A.n_rows) return;
  int expert = 0;
  if (A.offsets) {
    expert = expert_of(A.offsets, A.n_experts, row);
    if (expert < 0) return;
  }
  __shared__ float factor[C % 28 == 0 ? 784 : 1];
  if constexpr (C % 28 == 0) stage28<THR>(factor, A.q28 + int64_t(expert) * 784, tid);
  const Products products(A, row, expert);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int at = 512 * (wave + WAVES * n), j = at + 8 * octet_of(lane);
    if (at >= d) break;  // (uniform over the wave)
    float v[8] = {};
    if (j < d) products.sum8(j, v);
    inside_column<1, FULL>(v, lane, cols);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int q = at + quad_at<false, FULL>(lane, h);
      if (q < d)
        *reinterpret_cast<float4*>(buf + q) =
            make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]);
    }
  }
  __syncthreads();
  const float unit = (A.row_unit ? A.row_unit[row] : 1.f) * A.turn.norm;
  if constexpr (C % 28 == 0) {
    float q[14];
    load28<true>(q, factor, lane);
    mix28<C / 28>(buf, A.turn.m, q, wave, WAVES, lane, [&](int i, float v) { buf[i] = v; });
    __syncthreads();
    const int half = cols / 2;  // (a power of two from 4 on)
    finish_row<T>(A, buf, row, expert, unit, 2 * (tid & (half - 1)), tid / half, THR / half, 0,
                  d);
  } else {
    const int p = 2 * tid;
    if (p >= cols) return;
    float u[C], w[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const float2 f = *reinterpret_cast<const float2*>(buf + c * cols + p);
      u[c] = f.x, w[c] = f.y;
    }
    across_columns<C>(u, w, [&](int c, float a, float b) {
      *reinterpret_cast<float2*>(buf + c * cols + p) = make_float2(a, b);
    });
    finish_row<T>(A, buf, row, expert, unit, p, 0, 1, 0, d);  // (of what this thread has put there)
  }
}

// A few rows of 28 m: four workgroups to a row, 7 segments each, where one to a row would leave most
// CUs idle. Each sums all products of the row, so the factor comes first here: 16 x 16 tiles of it on
// the matrix cores take a workgroup's 7 rows of the factor. Rows of 14336: 16 of them 11.0 us, where
// one workgroup each takes 14.5; 32 of them 12.4 and 14.5; 64 of them 17.5 and 14.8, so that half of
// the CUs is the limit.
constexpr int PARTS = 4;
template <typename T, int B>
__global__ __launch_bounds__(1024) void linear_out_part(LinearOut A) {
  extern __shared__ __attribute__((aligned(16))) float buf[];  // the row, then the 7 segments
  __shared__ float factor[784];
  constexpr int WAVES = 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int d = int(A.d_out), cols = A.turn.cols, m = A.turn.m;
  const int64_t row = blockIdx.x / PARTS;
  const int first = 7 * int(blockIdx.x % PARTS);  // segment
  int expert = 0;
  if (A.offsets) {
    expert = expert_of(A.offsets, A.n_experts, row);
    if (expert < 0) return;
  }
  stage28<1024>(factor, A.q28 + int64_t(expert) * 784, tid);
  const Products products(A, row, expert);
#pragma unroll 1
  for (int j = 8 * tid; j < d; j += 8192) {
    float v[8];
    products.sum8(j, v);
    *reinterpret_cast<float4*>(buf + j) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(buf + j + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
  __syncthreads();
  {
    const int n = lane & 15, quad = lane >> 4;
    float q[7];
#pragma unroll
    for (int s = 0; s < 7; ++s) q[s] = factor[(4 * s + quad) * 28 + first + (n < 7 ? n : 6)];
    // (in place: a wave reads all of its 16 places before it writes them)
    for (int p0 = 16 * wave; p0 < cols; p0 += 16 * WAVES) {
      const int p = p0 + n, pc = p < cols ? p : cols - 1;
      f32x4_t o[B] = {};
#pragma unroll
      for (int b = 0; b < B; ++b)
#pragma unroll
        for (int s = 0; s < 7; ++s)
          o[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(q[s], buf[(4 * s + quad) * m + 512 * b + pc],
                                                      o[b], 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int a = 4 * quad + r;
        if (a >= 7 || p >= cols) continue;
        if constexpr (B == 2) {
          buf[a * m + p] = o[0][r] + o[1][r];
          buf[a * m + p + 512] = o[0][r] - o[1][r];
        } else {
          buf[a * m + p] = o[0][r];
        }
      }
    }
  }
  __syncthreads();
  for (int at = 512 * wave; at < 7 * m; at += 512 * WAVES) {  // (uniform over the wave)
    const int j = at + 8 * octet_of(lane);
    float v[8] = {};
    if (j < 7 * m) load8(buf + j, v);
    const bool full = cols == 512;
    if (full)
      inside_column<1, true>(v, lane, cols);
    else
      inside_column<1, false>(v, lane, cols);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int q = at + (full ? quad_at<false, true>(lane, h) : quad_at<false, false>(lane, h));
      if (q < 7 * m)
        *reinterpret_cast<float4*>(buf + q) =
            make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]);
    }
  }
  __syncthreads();
  const float unit = (A.row_unit ? A.row_unit[row] : 1.f) * A.turn.norm;
  const int half = cols / 2;  // (a power of two from 4 on)
  finish_row<T>(A, buf, row, expert, unit, 2 * (tid & (half - 1)), tid / half, 1024 / half,
                first * m, 7 * m);
}

// Rows without a transform, and transforms whose columns are shorter than an octet (cols: 1, 2 or 4
// elements in each of 28 or fewer columns: the dense product).
template <typename T>
__global__ __launch_bounds__(256) void linear_out_any(LinearOut A) {
  __shared__ float small[128];
  const int tid = threadIdx.x, d = int(A.d_out);
  const int64_t row = workgroup();
  if (row >= A.n_rows) return;
  int expert = 0;
  if (A.offsets) {
    expert = expert_of(A.offsets, A.n_experts, row);
    if (expert < 0) return;
  }
  const float up = (A.row_unit ? A.row_unit[row] : 1.f) * A.turn.norm;
  const float* const mul = A.mul ? A.mul + int64_t(expert) * d : nullptr;
  const float* const bias = A.bias ? A.bias + int64_t(expert) * d : nullptr;
  const T* const res = A.residual ? static_cast<const T*>(A.residual) + row * A.ldr : nullptr;
  T* const y = static_cast<T*>(A.y) + row * A.ldy;
  const Products products(A, row, expert);
  constexpr int K = 4;
  for (int j = tid; j < d; j += 256 * K) {
    float v[K];
    products.sum_each<K>(j, 256, d, v);
    if (A.turn.rotate) {
      small[j] = v[0];  // (d <= 28 * 4)
      break;
    }
#pragma unroll 1
    for (int k = 0; k < K; ++k) {
      const int at = j + 256 * k;
      if (at < d) store1<T>(y, at, finish<T>(v[0] * up, at, mul, bias, res, A.act));
#pragma unroll
      for (int i = 1; i < K; ++i) v[i - 1] = v[i];
    }
  }
  if (!A.turn.rotate) return;
  __syncthreads();
  const float* q = A.q28 + int64_t(expert) * 784;
  for (int j = tid; j < d; j += 256) {
    const int a = j / A.turn.m, b = j % A.turn.m;
    float v = 0.f;
    for (int k = 0; k < d; ++k) {
      const float h = (__popc(unsigned(b & (k % A.turn.m))) & 1) ? -small[k] : small[k];
      v = fmaf(A.turn.has28 ? q[(k / A.turn.m) * 28 + a] : 1.f, h, v);
    }
    store1<T>(y, j, finish<T>(v * up, j, mul, bias, res, A.act));
  }
}

template <typename T>
int in_typed(const LinearIn& a, hipStream_t s) {
  const int cc = a.turn.rotate ? int(a.d_in / a.turn.cols) : 0;
  const int64_t table_blocks = a.table ? cdiv(a.w_rows, TABLE_ROWS) : 0;
  const int64_t lead = cdiv(table_blocks + (a.offsets ? 1 : 0), 8) * 8;
  const dim3 grid = grid_of(lead + cdiv(a.n_rows, 256) * 256);
#define KQ_IN(C_, N_, F_)                                                                            \
  launch("linear_in", linear_in<T, C_, N_, F_>, grid, dim3(in_threads(C_)), C_ ? size_t(a.d_in) * 4 : 0, s, a, \
         int(table_blocks), int(lead))
  if (!a.turn.rotate) {
    const int64_t n = cdiv(a.d_in, 2048);
    return n <= 1 ? KQ_IN(0, 1, false) : n <= 2 ? KQ_IN(0, 2, false) : n <= 4 ? KQ_IN(0, 4, false) : n <= 8 ? KQ_IN(0, 8, false)
                                                                                  : KQ_IN(0, 16, false);
  }
  const bool full = a.turn.cols == 512;
  switch (cc) {
    case 1:
      return full ? KQ_IN(1, 1, true) : KQ_IN(1, 1, false);
    case 2:
      return KQ_IN(2, 1, true);
    case 4:
      return KQ_IN(4, 1, true);
    case 8:
      return KQ_IN(8, 2, true);
    case 16:
      return KQ_IN(16, 4, true);
    case 32:
      return KQ_IN(32, 8, true);
    case 64:
      return KQ_IN(64, 16, true);
    case 28:
      return full ? KQ_IN(28, 2, true) : KQ_IN(28, 2, false);
    default:
      return KQ_IN(56, 4, true);
  }
#undef KQ_IN
}

template <typename T>
int out_typed(LinearOut a, hipStream_t s) {
  // two neighbours at once where every row of each operand begins on two
  const size_t pair = 2 * sizeof(T);
  a.pairs = aligned(a.y, pair) && a.ldy % 2 == 0 && aligned(a.bias, 8) &&
            (!a.residual || (aligned(a.residual, pair) && a.ldr % 2 == 0));
  const dim3 grid = grid_of(a.n_rows);
  if (!a.turn.rotate || a.turn.cols < 8)
    return launch("linear_out", linear_out_any<T>, grid, dim3(256), 0, s, a);
#define KQ_OUT(C_, F_) \
  launch("linear_out", linear_out<T, C_, F_>, grid, dim3(threads(C_)), size_t(a.d_out) * 4, s, a)
  if (a.turn.has28 && a.n_rows * PARTS <= device_cus() / 2) {
    const dim3 parts(static_cast<unsigned>(a.n_rows * PARTS));
    return a.turn.m == 1024
               ? launch("linear_out", linear_out_part<T, 2>, parts, dim3(1024),
                        size_t(a.d_out) * 4, s, a)
               : launch("linear_out", linear_out_part<T, 1>, parts, dim3(1024),
                        size_t(a.d_out) * 4, s, a);
  }
  const bool full = a.turn.cols == 512;
  switch (a.d_out / a.turn.cols) {
    case 1:
      return full ? KQ_OUT(1, true) : KQ_OUT(1, false);
    case 2:
      return KQ_OUT(2, true);
    case 4:
      return KQ_OUT(4, true);
    case 8:
      return KQ_OUT(8, true);
    case 16:
      return KQ_OUT(16, true);
    case 32:
      return KQ_OUT(32, true);
    case 64:
      return KQ_OUT(64, true);
    case 28:
      return full ? KQ_OUT(28, true) : KQ_OUT(28, false);
    default:
      return KQ_OUT(56, true);
  }
#undef KQ_OUT
}

}  // namespace

LinearTurn linear_turn(int64_t d, bool rotate) {
  const RotDim rd = rot_dim(d);
  LinearTurn t{rotate, rotate && rd.has28, 1, 1, 1.f};
  if (rotate) {
    t.m = int(rd.m), t.cols = t.m < 512 ? t.m : 512;
    t.norm = float(1.0 / std::sqrt(double(rd.m)));
  }
  return t;
}

int linear_in_launch(const LinearIn& a, hipStream_t s) {
  return a.x_dtype == KRONQ_BF16 ? in_typed<uint16_t>(a, s) : in_typed<float>(a, s);
}
int linear_out_launch(const LinearOut& a, hipStream_t s) {
  return a.y_dtype == KRONQ_BF16 ? out_typed<uint16_t>(a, s) : out_typed<float>(a, s);
}

}  // namespace kq
