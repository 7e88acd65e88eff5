// The served layer on any number of rows (tokens), with bias, activation and residual in its
// epilogue, and its form for a mixture of experts:
//   x' = T_in diag(mul_in) x,  y' = W_hat' x',  y = act(diag(mul_out) T_out y' + bias) + residual,
// W_hat' = scale (code - zero) per row and group of columns, T the Hadamard factors of the online
// transforms. Up to four rows of one layer go through the byte digits of online_gemv_mfma (whose
// matrix instructions have room for no more); otherwise three launches:
//   1. linear_in: x' as fp16 in MFMA-fragment order, each row scaled by a power of two of its own
//      that brings its largest value into [2^7, 2^8); beside it the tables of the weights' scales
//      and zeros, and for experts the list of row tiles.
//   2. linear_few or, for many rows, linear_ring: products of 32 rows and 32 rows of W_hat' on
//      v_mfma_f32_32x32x16_f16. A lane takes the packed codes of its own weight row and spreads them
//      to fp16 in registers.
//   3. linear_out: the transform of y', and the epilogue.
// Weights enter the matrix products in one of two forms (SCALED below): as fp16 s (c - z), each row
// of W divided by a power of two, from a table of fp16 scales and zeros that linear_in prepares
// (many rows of x: an AND, an addition and a multiplication a pair of codes are all there is to do); or
// as the exact integers c - z, each group's sum taking its fp32 scale (few rows, where the table would
// cost more than the sums, and fp32 outputs).
// Precision. For bf16 outputs x' (and with the table s, and its product with the exact c - z) is rounded
// to fp16, 2^-11 against the output's own 2^-8, and summed in fp32, parts of split columns included (as
// fp16 they were 2% faster for 8192 rows). For fp32 outputs x' is held in two fp16 planes (value and
// rest: 22 bits, and never coarser than 2^-32 of the row's largest value) and the weights are exact.
#include <cmath>
#include <type_traits>

#include "kq_linear.hpp"

namespace kq {
namespace {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
#define KQ_RSRC(base, bytes) \
  __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(static_cast<const void*>(base)), 0, int(bytes), \
                                    0x00027000)
#define KQ_LDS(p) ((__attribute__((address_space(3))) void*)(p))

using Tile = LinearTile;

// tiles that any offsets of n_experts over n_rows rows can give: the experts' ranges overlap at
// most n_rows / 32 + 1 units once and one more for each expert after the first, and each expert's
// last tile may be short
__host__ __device__ inline int64_t most_tiles(int64_t n_rows, int64_t n_experts, int nt) {
  const int64_t e = n_experts < n_rows ? n_experts : n_rows;
  return (cdiv(n_rows, 32) + e - 1) / nt + e;
}

constexpr int BLOCK = LINEAR_BLOCK;

// ---- 2. products ---------------------------------------------------------------------------------
struct MmArgs {
  const uint32_t* packed;
  int64_t ldp, d_out, w_rows;
  const uint16_t* xf;
  int64_t plane;
  int ng;             // groups of 128 columns
  const uint32_t* table;  // SCALED
  const float *scales, *zeros;  // otherwise
  int64_t ldsz;
  int gpq;
  const Tile* tiles;  // null: one layer, unit tiles in order
  int64_t n_rows;
  int row_blocks;
  float* part;        // [row][ld]
  int64_t ld;
  float* kept;        // [worker][32 NT][rows of W of an item]
};

__device__ __forceinline__ f16x2_t h2(uint32_t v) { return __builtin_bit_cast(f16x2_t, v); }
__device__ __forceinline__ uint32_t u2(f16x2_t v) { return __builtin_bit_cast(uint32_t, v); }

// eight 3-bit codes of a 24-bit field, codes 0-3 from bit 0 on and 4-7 from bit 16 on
__device__ __forceinline__ uint32_t halves3(uint32_t g) {
  return (g & 0xFFFu) | ((g << 4) & 0x0FFF0000u);
}
__device__ __forceinline__ uint32_t field3(const uint32_t* w, int jj) {
  switch (jj) {
    case 0:
      return w[0];
    case 1:
      return __builtin_amdgcn_alignbit(w[1], w[0], 24);
    case 2:
      return __builtin_amdgcn_alignbit(w[2], w[1], 16);
    default:
      return w[2] >> 8;
  }
}

// The eight codes of step jj of a chunk as fp16 weights s (c - z). A field of code bits at `shift` under
// 0x6400 is 1024 + c 2^shift, and adding -(1024 + z 2^shift) leaves (c - z) 2^shift exactly (|z| < 1024:
// a multiple of 2^shift below 2^11 of them), so that the product alone is rounded. (One fused
// multiply-add with -z s as fp16 saves an instruction a pair, and its rounding moves all weights of
// a group by the same amount: 8 bits and activations of mean 3, 6e-3 of the result.)
// sz: fp16 {s / unit, -(1024 + z)}.
template <int BITS>
__device__ __forceinline__ u32x4_t spread(const uint32_t* w, int jj, uint32_t sz) {
  const _Float16 s = h2(sz)[0], nz = h2(sz)[1];
  uint32_t base = 0x64006400u;
  asm("" : "+v"(base));  // (in a register, mask and base make one instruction)
  auto weights = [&](uint32_t v, int shift) {
    const float up = float(1 << shift);
    const _Float16 t = s * _Float16(1.f / up);
    const _Float16 n =
        shift ? __builtin_elementwise_fma(nz, _Float16(up), _Float16(1024.f * (up - 1.f))) : nz;
    return u2((h2(v | base) + f16x2_t{n, n}) * f16x2_t{t, t});
  };
  if constexpr (BITS == 2) {
    const uint32_t v = w[jj >> 1] >> (8 * (jj & 1)), v4 = v >> 4;
    return u32x4_t{weights(v & 0x00030003u, 0), weights(v & 0x000C000Cu, 2),
                   weights(v4 & 0x00030003u, 0), weights(v4 & 0x000C000Cu, 2)};
  } else if constexpr (BITS == 3) {
    const uint32_t v = halves3(field3(w, jj)), v6 = v >> 6;
    return u32x4_t{weights(v & 0x00070007u, 0), weights(v & 0x00380038u, 3),
                   weights(v6 & 0x00070007u, 0), weights(v6 & 0x00380038u, 3)};
  } else if constexpr (BITS == 4) {
    const uint32_t v = w[jj], v8 = v >> 8;
    return u32x4_t{weights(v & 0x000F000Fu, 0), weights(v & 0x00F000F0u, 4),
                   weights(v8 & 0x000F000Fu, 0), weights(v8 & 0x00F000F0u, 4)};
  } else {
    const uint32_t a = w[2 * jj], b = w[2 * jj + 1];
    return u32x4_t{weights(a & 0x00FF00FFu, 0), weights((a >> 8) & 0x00FF00FFu, 0),
                   weights(b & 0x00FF00FFu, 0), weights((b >> 8) & 0x00FF00FFu, 0)};
  }
}

// The same codes as the exact integers c - z: 0x6400 | c is 1024 + c; nz = fp16 pair of -(1024 + z).
template <int BITS>
__device__ __forceinline__ u32x4_t spread_int(const uint32_t* w, int jj, uint32_t nz) {
  auto add = [&](uint32_t v) { return u2(h2(v | 0x64006400u) + h2(nz)); };
  if constexpr (BITS == 2) {
    const uint32_t v = w[jj >> 1] >> (8 * (jj & 1));
    return u32x4_t{add(v & 0x00030003u), add((v >> 2) & 0x00030003u), add((v >> 4) & 0x00030003u),
                   add((v >> 6) & 0x00030003u)};
  } else if constexpr (BITS == 3) {
    const uint32_t v = halves3(field3(w, jj));
    return u32x4_t{add(v & 0x00070007u), add((v >> 3) & 0x00070007u), add((v >> 6) & 0x00070007u),
                   add((v >> 9) & 0x00070007u)};
  } else if constexpr (BITS == 4) {
    const uint32_t v = w[jj];
    return u32x4_t{add(v & 0x000F000Fu), add((v >> 4) & 0x000F000Fu), add((v >> 8) & 0x000F000Fu),
                   add((v >> 12) & 0x000F000Fu)};
  } else {
    const uint32_t a = w[2 * jj], b = w[2 * jj + 1];
    return u32x4_t{add(a & 0x00FF00FFu), add((a >> 8) & 0x00FF00FFu), add(b & 0x00FF00FFu),
                   add((b >> 8) & 0x00FF00FFu)};
  }
}

__device__ __forceinline__ f32x16_t mfma(u32x4_t a, u32x4_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a),
                                                __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

template <int N>
__device__ __forceinline__ void wait_vm() {  // s_waitcnt vmcnt(N), the other counters free
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

// this lane's codes of a group: two chunks of 32
template <int BITS>
__device__ __forceinline__ void load_codes(uint32_t* w, const uint32_t* p) {
  if constexpr (BITS == 3) {
#pragma unroll
    for (int k = 0; k < 6; k += 2) {
      const uint2 v = *reinterpret_cast<const uint2*>(p + k);
      w[k] = v.x, w[k + 1] = v.y;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 2 * BITS; k += 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(p + k);
      w[k] = v.x, w[k + 1] = v.y, w[k + 2] = v.z, w[k + 3] = v.w;
    }
  }
}

// Few rows: the codes' way from memory bounds it. A workgroup of eight waves, one per CU, takes 256
// rows of W (32 a wave) and a tile of NT units; everything comes straight to LDS in whole lines, and
// the lanes take their own rows' codes from there. (Codes that each lane loads from its own row are
// one L1 access a lane: those bound it, 66 us for 8 experts of 14336 x 4096 at 4 bits with 32 rows
// that take 52 this way, at 3.3 TB/s of what has to be read.) In LDS:
//   x': RG groups of NP pieces (unit, plane) of 8 KB in fragment order, one step of 16 columns a wave;
//   codes: CB batches of BG groups, of LB bytes a row: with rows of 128 bytes piece p of 16 stands at
//     p ^ (row & 7), so that eight lanes reading theirs meet in no bank;
//   scales and zeros: two sets of four groups, [row][group].
// One barrier a group, in its middle: it publishes the next group's operands and frees those of the
// group before, which the loads after it then fill. vmcnt counts in order, and the loads below leave in
// an order that is the same for every group of a batch, so `newer` tells at compile time how many may
// still be out; loads past the end of the range leave too (out of bounds: they read nothing).
constexpr int newer(int u, int np, int rg, int cb, int bg, int cl) {  // group u of a batch
  int x = 0, c = 0;  // loads that left after those of the next group's x', and of its codes
  for (int back = rg - 2; back >= 1; --back)  // (the middle of the group `back` groups ago)
    x += (back < rg - 2 ? np : 0) + ((u - back) % bg == 0 ? cl : 0);  // (codes after x')
  for (int back = (cb - 1) * bg - 2; back >= 1; --back) c += np + ((u - back) % bg == 0 ? cl : 0);
  return u == bg - 1 && c < x ? c : x;
}

template <int BITS, int NT, int PLANES>
__global__ __launch_bounds__(512, 2) void linear_few(MmArgs A) {
  constexpr int NP = NT * PLANES, XG = NP * 2048;  // (dwords of a group of x')
  constexpr int RG = NP == 1 ? 4 : 3, CB = 3;
  constexpr int LB = BITS == 3 ? 96 : 128, PPR = LB / 16, BG = LB / (16 * BITS);
  constexpr int CL = BLOCK * PPR / 512;  // loads of a batch of codes per wave
  constexpr int CODES = RG * XG, PARAMS = CODES + CB * BLOCK * LB / 4, SET = BLOCK * 4 * 2;
  __shared__ __attribute__((aligned(16))) uint32_t lds[PARAMS + 2 * SET];
  static_assert(sizeof(lds) <= 163840, "160 KB a CU");
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // (workers that share an XCD stand next to one another in the deal, as below)
  const int W = int(gridDim.x), id = int(blockIdx.x & 7) * (W >> 3) + int(blockIdx.x >> 3);
  const int ntiles = A.tiles ? A.tiles[0].expert : int(cdiv(A.n_rows, 32 * NT));
  const int items = ntiles * A.row_blocks;
  const LinearDeal deal = linear_deal(items, A.ng, W);
  const int rest = items - deal.full * W;
  int round = 0, ua = id * deal.per;  // next group of the rest
  const int ub = ua + deal.per < rest * A.ng ? ua + deal.per : rest * A.ng;
  for (;;) {
    int item, g0 = 0, g1 = A.ng;
    if (round < deal.full) {
      item = round++ * W + id;
    } else if (ua < ub) {
      const int r = ua / A.ng;
      item = deal.full * W + r;
      g0 = ua - r * A.ng;
      g1 = g0 + (ub - ua) < A.ng ? g0 + (ub - ua) : A.ng;
      ua += g1 - g0;
    } else {
      break;
    }
    const int rb = item % A.row_blocks, ti = item / A.row_blocks;
    const Tile t = A.tiles ? A.tiles[1 + ti] : Tile{0, ti * NT, 0, int(A.n_rows)};
    const int last = (t.hi - 1) >> 5;  // last unit
    const int ngr = g1 - g0;
    const int64_t row0 = int64_t(t.expert) * A.d_out + int64_t(rb) * BLOCK;  // of W
    const int left = int(A.d_out - int64_t(rb) * BLOCK);
    const int n_last = (left < BLOCK ? left : BLOCK) - 1;  // last row of W here
    // x'
    auto issue_x = [&](int g) {  // past the end: the last group again, never read
      const int at = ((g0 + (g < ngr ? g : ngr - 1)) * 8 + wave) * 1024;
      uint32_t* const dst = lds + (g % RG) * XG + wave * 256;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const int un = t.unit + p / PLANES;
        const uint16_t* const rows =
            A.xf + (p % PLANES) * A.plane + (un < last ? un : last) * int64_t(A.ng) * 4096;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(KQ_RSRC(rows, A.ng * 8192), KQ_LDS(dst + p * 2048), 16,
                                                 lane * 16, at, 0, 0);
      }
    };
    // codes
    const auto code_src = KQ_RSRC(A.packed + row0 * A.ldp,
                               (int64_t(n_last) * A.ldp + A.ng * 4 * BITS) * 4);
    int code_at[CL];
#pragma unroll
    for (int i = 0; i < CL; ++i) {
      const int idx = i * 512 + tid, n = idx / PPR, slot = idx % PPR;
      const int piece = PPR == 8 ? slot ^ (n & 7) : slot;
      code_at[i] = (n < n_last ? n : n_last) * int(A.ldp * 4) + g0 * 16 * BITS + piece * 16;
    }
    auto issue_codes = [&](int b) {
      uint32_t* const dst = lds + CODES + ((b + CB) % CB) * (BLOCK * LB / 4) + wave * 256;
      const bool in = b >= 0 && b * BG < ngr;
#pragma unroll
      for (int i = 0; i < CL; ++i) {
        const int at = in ? code_at[i] + b * LB : -256;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(code_src, KQ_LDS(dst + i * 2048), 16, at, 0, 0, 0);
      }
    };
    // scales and zeros of groups g to g + 3
    const int szn = (n_last * int(A.ldsz) + A.ng / A.gpq) * 4;
    const auto s_src = KQ_RSRC(A.scales + row0 * A.ldsz, szn), z_src = KQ_RSRC(A.zeros + row0 * A.ldsz, szn);
    auto issue_params = [&](int g) {
      uint32_t* const dst = lds + PARAMS + ((g >> 2) & 1) * SET + wave * 64;
      const int k = g + (tid & 3);
      const unsigned q = unsigned(g0 + (k < ngr ? k : ngr - 1)) / unsigned(A.gpq);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int n = i * 128 + (tid >> 2);
        const int at = (n < n_last ? n : n_last) * int(A.ldsz * 4) + int(q) * 4;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(s_src, KQ_LDS(dst + i * 512), 4, at, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(z_src, KQ_LDS(dst + 1024 + i * 512), 4, at, 0, 0, 0);
      }
    };
    // what a lane takes of a group: its row's codes of half of the columns (two chunks of 32), scale and
    // fp16 pair of -(1024 + zero)
    const int mine = 32 * wave + (lane & 31), h = lane >> 5;
    auto read_codes = [&](uint32_t (&w)[2 * BITS], int g, auto kc) {  // kc: group of its batch
      constexpr int k = decltype(kc)::value;
      const uint32_t* const c = lds + CODES + (g / BG % CB) * (BLOCK * LB / 4) + mine * (LB / 4);
      if constexpr (BITS == 3) {
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const u32x2_t v = *reinterpret_cast<const u32x2_t*>(c + k * 12 + h * 6 + 2 * i);
          w[2 * i] = v[0], w[2 * i + 1] = v[1];
        }
      } else {
#pragma unroll
        for (int i = 0; i < BITS / 2; ++i) {
          const int piece = k * BITS + h * (BITS / 2) + i;
          const u32x4_t v = *reinterpret_cast<const u32x4_t*>(c + 4 * (piece ^ (mine & 7)));
#pragma unroll
          for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
        }
      }
    };
    auto read_params = [&](float& s, uint32_t& nz, int g) {
      const uint32_t* const c = lds + PARAMS + ((g >> 2) & 1) * SET + mine * 4 + (g & 3);
      s = __uint_as_float(c[0]);
      const _Float16 z = _Float16(-1024.f - __uint_as_float(c[1024]));
      nz = u2(f16x2_t{z, z});
    };
    u32x4_t a[2][NP];
    auto frags = [&](int g, int q) {
      const uint32_t* const buf = lds + (g % RG) * XG + lane * 4 + q * 256;
#pragma unroll
      for (int i = 0; i < NP; ++i) a[q & 1][i] = *reinterpret_cast<const u32x4_t*>(buf + i * 2048);
    };
    f32x16_t acc[NT] = {}, sum[NT] = {};
    uint32_t cw[2 * BITS], cw1[2 * BITS], sz, sz1;
    float sc, sc1;
    auto group = [&](int g, auto uc) {
      constexpr int u = decltype(uc)::value;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        if (q == 4) {
          wait_vm<newer(u, NP, RG, CB, BG, CL)>();
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
          issue_x(g + RG - 1);
          __builtin_amdgcn_sched_barrier(0);  // (the order that `newer` counts on)
          if constexpr (u == 0) issue_codes(g / BG + CB - 1);
          __builtin_amdgcn_sched_barrier(0);
          if ((g & 3) == 0) issue_params(g + 4);
          __builtin_amdgcn_sched_barrier(0);
          read_codes(cw1, g + 1, std::integral_constant<int, (u + 1) % BG>{});
          read_params(sc1, sz1, g + 1);
        }
        frags(q < 7 ? g : g + 1, (q + 1) & 7);
        const u32x4_t b = spread_int<BITS>(cw + (q >> 2) * BITS, q & 3, sz);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          if constexpr (PLANES == 2) sum[i] = mfma(a[q & 1][2 * i + 1], b, sum[i]);
          sum[i] = mfma(a[q & 1][PLANES * i], b, sum[i]);
        }
        __builtin_amdgcn_sched_barrier(0);  // (else every step's operands are read at once)
      }
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[i][k] = fmaf(sc, sum[i][k], acc[i][k]), sum[i][k] = 0.f;
#pragma unroll
      for (int k = 0; k < 2 * BITS; ++k) cw[k] = cw1[k];
      sc = sc1, sz = sz1;
    };
    issue_params(0);
    __builtin_amdgcn_sched_barrier(0);
    // (the loads of the middles before the first group)
    constexpr int FIRST = RG - 1 > (CB - 1) * BG ? RG - 1 : (CB - 1) * BG;
#pragma unroll
    for (int s = -FIRST; s < 0; ++s) {
      if (s + RG - 1 >= 0) issue_x(s + RG - 1);
      __builtin_amdgcn_sched_barrier(0);
      if (s % BG == 0) issue_codes(s / BG + CB - 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    wait_vm<newer(BG - 1, NP, RG, CB, BG, CL)>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read_codes(cw, 0, std::integral_constant<int, 0>{});
    read_params(sc, sz, 0);
    frags(0, 0);
    for (int g = 0; g < ngr; g += BG) {
      group(g, std::integral_constant<int, 0>{});
      if constexpr (BG > 1) {
        if (g + 1 < ngr) group(g + 1, std::integral_constant<int, 1>{});
      }
      if constexpr (BG > 2) {
        if (g + 2 < ngr) group(g + 2, std::integral_constant<int, 2>{});
        if (g + 3 < ngr) group(g + 3, std::integral_constant<int, 3>{});
      }
    }
    wait_vm<0>();  // (loads past the end still write to LDS)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    // a worker that began inside an item keeps its part
    const int64_t ld = g0 > 0 ? BLOCK : A.ld, n = int64_t(rb) * BLOCK + mine;
    float* const part =
        g0 > 0 ? A.kept + (int64_t(id) * NT - t.unit) * 32 * BLOCK - rb * BLOCK : A.part;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int mu = (t.unit + i) * 32, m0 = mu + 4 * h;
      float* p = part + int64_t(m0) * ld + n;
      const bool whole = mu >= t.lo && mu + 32 <= t.hi;  // (uniform) every row of it is the tile's
      if (mine > n_last) continue;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const int m = m0 + 8 * (k >> 2) + (k & 3);
        if (whole || (m >= t.lo && m < t.hi)) *p = acc[i][k];
        p += (k & 3) == 3 ? 5 * ld : ld;
      }
    }
  }
}

// Many rows. A workgroup of four waves takes 128 RT rows of W (32 RT a wave) and a tile of NT units of rows of
// x'; a lane holds the codes of RT rows of W and half of the columns, 64 of them a stage. x' comes
// through LDS: a stage is 64 columns (half a group, a chunk of each lane's codes) of NT units in
// PLANES planes, pieces of 4 KB that the waves bring straight to LDS, in fragment order as they
// stand, through a ring of R stages. One barrier a stage, in its middle: it publishes the next stage
// and frees the buffer of the one before, which the loads of R - 1 stages on then fill; operands are
// read one step of 16 columns ahead.
//   SCALED, NT = 4, RT = 2 (many rows): the matrix instructions bound it. Two workgroups per CU (64 KB
//     of LDS and 256 registers a lane each), so that one wave's spreading of codes runs beside the
//     other's matrix instructions.
//   PLANES = 2, NT = 2, RT = 2: the same for fp32 results.
// 8192 rows of 4096 x 4096 at 4 bits: 250 us, 1.10 PFLOP/s, where a large plain matrix product reaches
// 1.22 to 1.32. A lane reads its row of W in batches; the fp32 scales and zeros (not SCALED) come
// through LDS eight groups at a time, since 32 rows lie in 32 lines of either.
template <int BITS, int NT, int PLANES, bool SCALED>
__global__ __launch_bounds__(256, 2) void linear_ring(MmArgs A) {
  constexpr int RT = BLOCK / 128;                        // units of 32 rows of W a wave
  constexpr int NP = NT * PLANES, STAGE = NP * 1024;     // (dwords)
  constexpr int R = 4;                                   // stages of the ring
  constexpr int BG = BITS == 2 ? 2 : 1;                  // groups of a batch of codes: 8 words a lane
  constexpr int SG = 8;  // groups of scales and zeros in LDS
  // the ring, then {scale, fp16 pair of -(1024 + zero)} by group and row (one array: with a second one
  // the compiler waits for all loads to LDS before each read)
  __shared__ __attribute__((aligned(16))) uint32_t lds[R * STAGE + (SCALED ? 0 : 2 * SG * BLOCK)];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Workers that share an XCD (workgroup % 8) stand next to one another in the deal, so that the x'
  // of a tile is read through one L2, by all blocks of W at about the same time.
  const int W = int(gridDim.x), id = int(blockIdx.x & 7) * (W >> 3) + int(blockIdx.x >> 3);
  const int ntiles = A.tiles ? A.tiles[0].expert : int(cdiv(A.n_rows, 32 * NT));
  const int items = ntiles * A.row_blocks;
  const LinearDeal deal = linear_deal(items, A.ng, W);
  const int rest = items - deal.full * W;
  int round = 0, ua = id * deal.per;  // next group of the rest
  const int ub = ua + deal.per < rest * A.ng ? ua + deal.per : rest * A.ng;
  for (;;) {
    int item, g0 = 0, g1 = A.ng;
    if (round < deal.full) {
      item = round++ * W + id;
    } else if (ua < ub) {
      const int r = ua / A.ng;
      item = deal.full * W + r;
      g0 = ua - r * A.ng;
      g1 = g0 + (ub - ua) < A.ng ? g0 + (ub - ua) : A.ng;
      ua += g1 - g0;
    } else {
      break;
    }
    const int rb = item % A.row_blocks, ti = item / A.row_blocks;
    const Tile t = A.tiles ? A.tiles[1 + ti] : Tile{0, ti * NT, 0, int(A.n_rows)};
    const int64_t n0 = int64_t(rb) * BLOCK + wave * (32 * RT);
    const int last = (t.hi - 1) >> 5;  // last unit
    const int nst = 2 * (g1 - g0);
    // this wave's piece of a stage, and the first of the NP of its four steps that it brings
    const int piece = wave % NP, step = wave / NP * NP, un = t.unit + piece / PLANES;
    // (buffer loads: beside global_load_lds the compiler waits for every outstanding load before it
    // uses one that went to a register)
    const uint16_t* const rows = A.xf + (piece % PLANES) * A.plane +
                                 (un < last ? un : last) * int64_t(A.ng) * 4096;
    const auto src = KQ_RSRC(rows, A.ng * 8192);
    auto issue = [&](int st) {  // past the end: the last stage again, never read
      const int at = (2 * g0 + (st < nst ? st : nst - 1)) * 4096;
      uint32_t* dst = lds + (st & (R - 1)) * STAGE + piece * 1024;
#pragma unroll
      for (int q = 0; q < NP; ++q)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(src, KQ_LDS(dst + (step + q) * 256), 16, lane * 16,
                                                 at + (step + q) * 1024, 0, 0);
    };
    const uint32_t* wp[RT];
    int64_t wr[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const int64_t n = n0 + 32 * i + (lane & 31);
      wr[i] = int64_t(t.expert) * A.d_out + (n < A.d_out ? n : A.d_out - 1);
      wp[i] = A.packed + wr[i] * A.ldp + (int64_t(g0) * 4 + (lane >> 5) * 2) * BITS;
    }
    const int ngr = g1 - g0;
    uint32_t cw[RT][BG * 2 * BITS], next[RT][BG * 2 * BITS];
    auto codes = [&](uint32_t (&w)[RT][BG * 2 * BITS], int gb) {  // the batch of the range's group gb
#pragma unroll
      for (int k = 0; k < BG; ++k)
#pragma unroll
        for (int i = 0; i < RT; ++i)
          load_codes<BITS>(w[i] + k * 2 * BITS,
                           wp[i] + int64_t(gb + k < ngr ? gb + k : ngr - 1) * 4 * BITS);
    };
    uint32_t sz[RT], sz1[RT];  // SCALED: of this group and the next one
    auto table = [&](int gi) {
      const int g = g0 + (gi < ngr ? gi : ngr - 1);
#pragma unroll
      for (int i = 0; i < RT; ++i) sz1[i] = A.table[int64_t(g) * A.w_rows + wr[i]];
    };
    // otherwise: this thread's row and four of the eight groups (per 128 rows)
    float sc[RT], ps[SCALED ? 1 : RT][4], pz[SCALED ? 1 : RT][4];
    const int64_t brow = int64_t(t.expert) * A.d_out + int64_t(rb) * BLOCK;
    auto fetch = [&](int gi) {
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const int r = int(threadIdx.x >> 1) + 128 * i;
        const int64_t n = int64_t(rb) * BLOCK + r;
        const int64_t at = (n < A.d_out ? brow + r : brow) * A.ldsz;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int g = gi + 4 * int(threadIdx.x & 1) + k;
          const unsigned q = unsigned(g0 + (g < ngr ? g : ngr - 1)) / unsigned(A.gpq);
          ps[i][k] = A.scales[at + q], pz[i][k] = A.zeros[at + q];
        }
      }
    };
    uint2* const params = reinterpret_cast<uint2*>(lds + R * STAGE);  // [group % SG][row]
    auto put = [&]() {
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const _Float16 nz = _Float16(-1024.f - pz[i][k]);
          params[(4 * (threadIdx.x & 1) + k) * BLOCK + (threadIdx.x >> 1) + 128 * i] =
              make_uint2(__float_as_uint(ps[i][k]), u2(f16x2_t{nz, nz}));
        }
    };
    f32x16_t acc[NT][RT] = {}, sum[SCALED ? 1 : NT][SCALED ? 1 : RT] = {};
    if constexpr (SCALED)
      table(0);
    else
      fetch(0);
    codes(cw, 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int st = 0; st < R - 1; ++st) issue(st);
    if constexpr (!SCALED) put();
    u32x4_t a[2][NP];
    auto frags = [&](int st, int q) {
      const uint32_t* buf = lds + (st & (R - 1)) * STAGE + lane * 4 + q * 256;
#pragma unroll
      for (int i = 0; i < NP; ++i) a[q & 1][i] = *reinterpret_cast<const u32x4_t*>(buf + i * 1024);
    };
    // stage u of a batch
    auto stage = [&](int st, auto uc) {
      constexpr int u = decltype(uc)::value, h = u & 1;
      const int gi = st >> 1;
      if constexpr (h == 0 && SCALED) {
#pragma unroll
        for (int i = 0; i < RT; ++i) sz[i] = sz1[i];
        table(gi + 1);
      }
      if constexpr (h == 0 && !SCALED) {
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          const uint2 v = params[(gi & (SG - 1)) * BLOCK + 32 * (RT * wave + i) + (lane & 31)];
          sc[i] = __uint_as_float(v.x), sz[i] = v.y;
        }
        if ((gi & (SG - 1)) == 0 && gi + SG < ngr) fetch(gi + SG);
      }
      // (every wave has read the last of the eight groups before the barrier of this group's first
      // stage, and reads the next one's after that of its second)
      if constexpr (h == 1 && !SCALED)
        if ((gi & (SG - 1)) == SG - 1 && gi + 1 < ngr) put();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (q == 2) {
          // the next stage's loads have landed (those of the R - 3 after it may be out)
          wait_vm<(R - 3) * NP>();
          if constexpr (h == 1 && !SCALED) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          __builtin_amdgcn_s_barrier();
          issue(st + R - 1);
          __builtin_amdgcn_sched_barrier(0);
        }
        frags(q < 3 ? st : st + 1, (q + 1) & 3);
        u32x4_t b[RT];
#pragma unroll
        for (int k = 0; k < RT; ++k)
          b[k] = SCALED ? spread<BITS>(cw[k] + u * BITS, q, sz[k])
                        : spread_int<BITS>(cw[k] + u * BITS, q, sz[k]);
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int k = 0; k < RT; ++k) {
            if constexpr (SCALED) {
              acc[i][k] = mfma(a[q & 1][i], b[k], acc[i][k]);
            } else {
              if constexpr (PLANES == 2) sum[i][k] = mfma(a[q & 1][2 * i + 1], b[k], sum[i][k]);
              sum[i][k] = mfma(a[q & 1][PLANES * i], b[k], sum[i][k]);
            }
          }
        __builtin_amdgcn_sched_barrier(0);  // (else every step's operands are read at once, and spill)
      }
      if constexpr (!SCALED) {
        if constexpr (h == 1) {
#pragma unroll
          for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int k = 0; k < RT; ++k)
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                acc[i][k][r] = fmaf(sc[k], sum[i][k][r], acc[i][k][r]);
                sum[i][k][r] = 0.f;
              }
        }
      }
    };
    wait_vm<(R - 2) * NP>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    frags(0, 0);
    for (int gb = 0; gb < ngr; gb += BG) {
      codes(next, gb + BG);
      auto pair = [&](auto kc) {
        constexpr int k = decltype(kc)::value;
        stage(2 * (gb + k), std::integral_constant<int, 2 * k>{});
        stage(2 * (gb + k) + 1, std::integral_constant<int, 2 * k + 1>{});
      };
      pair(std::integral_constant<int, 0>{});
      if constexpr (BG > 1) {
        if (gb + 1 < ngr) pair(std::integral_constant<int, 1>{});
      }
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int k = 0; k < BG * 2 * BITS; ++k) cw[i][k] = next[i][k];
    }
    wait_vm<0>();  // (loads past the end still write to LDS)
    __builtin_amdgcn_s_barrier();
    // a worker that began inside an item keeps its part
    const int64_t ld = g0 > 0 ? BLOCK : A.ld;
    float* const part =
        g0 > 0 ? A.kept + (int64_t(id) * NT - t.unit) * 32 * BLOCK - rb * BLOCK : A.part;
#pragma unroll
    for (int k = 0; k < RT; ++k) {
      const int64_t n = n0 + 32 * k + (lane & 31);
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const int mu = (t.unit + i) * 32, m0 = mu + 4 * (lane >> 5);
        float* p = part + int64_t(m0) * ld + n;
        const bool whole = mu >= t.lo && mu + 32 <= t.hi;  // (uniform) every row of it is the tile's
        if (n < A.d_out) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int m = m0 + 8 * (r >> 2) + (r & 3);
            if (whole || (m >= t.lo && m < t.hi)) *p = acc[i][k][r];
            p += (r & 3) == 3 ? 5 * ld : ld;
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
}

// ---- plan and launches ---------------------------------------------------------------------------
// Up to this many rows of one layer go through the byte digits of the GEMV.
constexpr int64_t GEMV_ROWS = 4, GEMV_INPUTS = 32768;

struct Plan {
  int planes, nt, workers;
  bool scaled, few;
  int64_t tiles, row_blocks;
};

Plan make_plan(int64_t d_out, int64_t d_in, int64_t n_rows, int64_t n_experts, int y_dtype) {
  Plan p;
  p.planes = y_dtype == KRONQ_BF16 ? 1 : 2;
  // A tile of 32 rows for up to 32 rows (of an expert); more rows share the spread codes in tiles of
  // 64, or of 128 with the table, which pays for itself late: one layer at 4 bits takes, in tiles of
  // 64 and of 128, 36 and 49 us for 256 rows of 4096 x 4096, 73 and 76 us for 256 rows of 14336 x
  // 4096, 126 and 111 us for 512 of these; 8 experts of 14336 x 4096 take 169 and 174 us for 64 rows
  // each, 204 and 184 us for 80 each. (Experts of one size: how many rows each has is known on the
  // device only, and the mean decides.)
  const int64_t rows = cdiv(n_rows, n_experts);
  p.scaled = p.planes == 1 && rows > (n_experts == 1 ? 256 : 64);
  p.nt = p.scaled ? 4 : rows > 32 ? 2 : 1;
  p.few = p.nt * p.planes < 4;
  p.tiles = n_experts == 1 ? cdiv(n_rows, 32 * p.nt) : most_tiles(n_rows, n_experts, p.nt);
  p.row_blocks = cdiv(d_out, BLOCK);
  p.workers = device_cus() / 8 * 8 * (p.few ? 1 : 2);
  return p;
}

struct Ws {
  uint16_t* xf;
  float *row_unit, *w_unit, *part, *kept;
  uint32_t* table;
  Tile* tiles;
  int2* first;
  size_t bytes;
};

Ws carve(void* ws, const Plan& p, int64_t d_out, int64_t d_in, int64_t n_rows, int64_t n_experts) {
  Carver cv(ws);
  Ws w;
  w.xf = cv.take<uint16_t>(size_t(p.planes) * size_t(cdiv(n_rows, 32) * 32) * size_t(d_in));
  w.row_unit = cv.take<float>(size_t(n_rows));
  w.part = cv.take<float>(size_t(n_rows) * size_t(cdiv(d_out, 8) * 8));
  w.kept = cv.take<float>(size_t(p.workers) * size_t(32 * p.nt) * size_t(BLOCK));
  const size_t w_rows = p.scaled ? size_t(n_experts) * size_t(d_out) : 0;
  w.w_unit = cv.take<float>(w_rows);
  w.table = cv.take<uint32_t>(w_rows * size_t(d_in / 128));
  w.tiles = cv.take<Tile>(size_t(p.tiles) + 1);
  w.first = cv.take<int2>(size_t(n_experts));
  w.bytes = align256(cv.used) + 256;
  return w;
}

template <int BITS>
int launch_mm(const MmArgs& a, const Plan& p, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(p.workers));
  if (p.scaled) return launch("linear_ring", linear_ring<BITS, 4, 1, true>, grid, dim3(256), 0, s, a);
  if (!p.few) return launch("linear_ring", linear_ring<BITS, 2, 2, false>, grid, dim3(256), 0, s, a);
#define KQ_FEW(NT_, PL_) launch("linear_few", linear_few<BITS, NT_, PL_>, grid, dim3(512), 0, s, a)
  return p.planes == 2 ? KQ_FEW(1, 2) : p.nt == 1 ? KQ_FEW(1, 1) : KQ_FEW(2, 1);
#undef KQ_FEW
}

}  // namespace

size_t linear_ws_bytes(int64_t d_out, int64_t d_in, int64_t n_rows, int64_t n_experts) {
  if (d_out <= 0 || d_in < 128 || n_rows <= 0 || n_experts <= 0) return 0;
  size_t most = n_experts == 1 && n_rows <= GEMV_ROWS ? online_ws_bytes(d_out, d_in, n_rows) : 0;
  for (int t : {KRONQ_BF16, KRONQ_FP32}) {
    const Plan p = make_plan(d_out, d_in, n_rows, n_experts, t);
    const size_t b = carve(nullptr, p, d_out, d_in, n_rows, n_experts).bytes;
    most = b > most ? b : most;
  }
  return most;
}

int linear_launch(const LinearJob& j, void* ws, hipStream_t s) {
  LinearOut o{};
  o.n_rows = j.n_rows, o.d_out = j.d_out, o.mul = j.mul_out, o.q28 = j.q28_out;
  o.turn = linear_turn(j.d_out, (j.flags & KRONQ_ROT_OUT) != 0);
  o.bias = j.bias, o.act = j.act, o.residual = j.residual, o.ldr = j.ldr;
  o.y = j.y, o.y_dtype = j.y_dtype, o.ldy = j.ldy;
  o.offsets = j.offsets, o.n_experts = int(j.n_experts);
  if (!j.offsets && j.n_rows <= GEMV_ROWS && j.n_rows * j.d_in <= GEMV_INPUTS) {
    float* yr;
    KQ_TRY(online_product_launch(j.packed, j.ldp, j.scales, j.zeros, j.ldsz, j.bits, j.group,
                                 j.d_out, j.d_in, j.mul_in, j.q28_in, j.flags, j.x, j.x_dtype,
                                 j.ldx, j.n_rows, ws, &yr, s));
    o.part = yr, o.ld = j.d_out;
    return linear_out_launch(o, s);
  }
  const Plan p = make_plan(j.d_out, j.d_in, j.n_rows, j.n_experts, j.y_dtype);
  const Ws w = carve(ws, p, j.d_out, j.d_in, j.n_rows, j.n_experts);
  LinearIn a{};
  a.x = j.x, a.x_dtype = j.x_dtype, a.ldx = j.ldx, a.n_rows = j.n_rows, a.d_in = j.d_in;
  a.mul = j.mul_in, a.q28 = j.q28_in, a.turn = linear_turn(j.d_in, (j.flags & KRONQ_ROT_IN) != 0);
  a.bits = j.bits, a.planes = p.planes, a.xf = w.xf, a.row_unit = w.row_unit;
  a.plane = cdiv(j.n_rows, 32) * 32 * j.d_in;
  a.table = p.scaled ? w.table : nullptr, a.w_unit = w.w_unit;
  a.scales = j.scales, a.zeros = j.zeros, a.ldsz = j.ldsz;
  a.gpq = j.group / 128, a.ng = int(j.d_in / 128), a.w_rows = j.n_experts * j.d_out;
  a.offsets = j.offsets, a.n_experts = int(j.n_experts), a.nt = p.nt;
  a.max_tiles = p.tiles, a.tiles = w.tiles, a.first = w.first;
  KQ_TRY(linear_in_launch(a, s));
  MmArgs m{};
  m.packed = j.packed, m.ldp = j.ldp, m.d_out = j.d_out, m.w_rows = a.w_rows;
  m.xf = w.xf, m.plane = a.plane, m.ng = a.ng, m.table = w.table;
  m.scales = j.scales, m.zeros = j.zeros, m.ldsz = j.ldsz, m.gpq = a.gpq;
  m.tiles = j.offsets ? w.tiles : nullptr, m.n_rows = j.n_rows;
  m.row_blocks = int(p.row_blocks);
  m.part = w.part, m.ld = cdiv(j.d_out, 8) * 8, m.kept = w.kept;
  KQ_TRY(j.bits == 2   ? launch_mm<2>(m, p, s)
         : j.bits == 3 ? launch_mm<3>(m, p, s)
         : j.bits == 4 ? launch_mm<4>(m, p, s)
                       : launch_mm<8>(m, p, s));
  o.part = w.part, o.ld = m.ld;
  o.row_unit = w.row_unit;
  o.workers = p.workers, o.ng = a.ng, o.nt = p.nt, o.row_blocks = m.row_blocks, o.kept = w.kept;
  o.items = int(p.tiles * p.row_blocks), o.w_unit = p.scaled ? w.w_unit : nullptr;
  if (j.offsets) o.tiles = w.tiles, o.first = w.first;
  return linear_out_launch(o, s);
}

}  // namespace kq
