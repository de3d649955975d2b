// matmul_w4.hip -- albireo_matmul_w4: products of bf16 or 8-bit rows with 4-bit weights and group scales.
#include <hip/hip_runtime.h>

#include <stdint.h>

#include <utility>

#include "albireo_decode.h"

namespace {

#include "common.h"
#include "rows.h"

struct W4Args {
  const unsigned char* x;
  const float* x_scale;
  const uint8_t* q;
  const unsigned char* scales;
  const uint8_t* zeros;
  unsigned char* out;
  int64_t ldx, ldq, lds, ldz, ldo;
  int64_t N;
  int32_t B, K, n_blocks, m_blocks;
  bool scale_bf16, out_bf16;
};

// ----------------------------------------------------------------------------------------------
// The product.
//
// A workgroup of four waves takes RN = (4 / WK) NT 16 weight rows and up to MT 16 rows of x.  Weights are the
// B operand of the matrix instructions, straight from memory to registers: a lane loads 16 bytes, 32 columns
// of one weight row, so the 64 lanes of a load cover 16 rows by 128 columns, and each 16-byte load feeds four
// (bf16) or two (8-bit) instructions.  x is the A operand, staged in LDS a chunk of KC columns at a time with
// the columns of every eight reordered to the order the nibbles come out of a dword, together with the sum of
// each group of its columns, the weights' scales and, with zero points, scale (8 - zero).
//   bf16: a nibble becomes 1 + q / 16 by putting its bits under the exponent of 1 (two columns at a time:
//         shift, and-or).  The sum of a group starts at -1.5 sum x, which takes 1 + 8 / 16 off every weight,
//         so it holds sum x (q - 8) / 16, and is added to the result times 16 scale.
//   8 bits: the nibbles of a dword are two operands of four bytes (and, shift-and); the sum starts at
//         -8 sum x and is exact; one conversion and one multiply-add per value and group.
// The loads of the next chunk (x, scales and weights) are in flight while a chunk is multiplied; LDS is
// double-buffered with one barrier per chunk.
// With WK = 4 the waves share their rows and each takes every fourth 128 columns, joined through LDS.
// ----------------------------------------------------------------------------------------------
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(1)));

constexpr int W4_NT = 256;  // threads per workgroup

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_full(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}

// Sum over aligned groups of L = 2, 4, 8 or 16 lanes (every lane receives it).
template <int L, class Add>
__device__ __forceinline__ uint32_t group_sum(uint32_t v, Add add) {
  v = add(v, dpp_full<0xb1>(v));                      // quad_perm 1,0,3,2
  if constexpr (L >= 4) v = add(v, dpp_full<0x4e>(v));   // quad_perm 2,3,0,1
  if constexpr (L >= 8) v = add(v, dpp_full<0x141>(v));  // row_half_mirror
  if constexpr (L >= 16) v = add(v, dpp_full<0x140>(v)); // row_mirror
  return v;
}

// a's upper 32 lanes against b's lower 32
__device__ __forceinline__ void swap32(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
// a's odd rows of 16 lanes against b's even ones
__device__ __forceinline__ void swap16(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

template <bool I8, int G, int MT, int NT, int WK, int KC>
struct W4Shape {
  static constexpr int ROWS = MT * 16;             // rows of x
  static constexpr int RN = (4 / WK) * NT * 16;    // weight rows
  static constexpr int KS = KC / 128 / WK;         // 128-column steps of a chunk, per wave
  static constexpr int NG = KC / G;                // groups of a chunk
  static constexpr int ES = I8 ? 1 : 2;
  static constexpr int XST = KC * ES + 16;         // bytes from one LDS row of x to the next: 16 past a multiple of 256
  static constexpr int XU = ROWS * KC * ES / 16;   // 16-byte units of x in a chunk
  static constexpr int XPT = XU / W4_NT;           // per thread
  static constexpr int SPT = (RN * NG + W4_NT - 1) / W4_NT;  // scales per thread
  static_assert(XU % W4_NT == 0, "whole units per thread");
  struct Buf {
    alignas(16) unsigned char x[ROWS * XST];
    alignas(16) float sum[NG][ROWS];               // sum of x over a group (8 bits: its integer's value)
    alignas(16) float scale[NG][RN];
    alignas(16) float off[NG][RN];                 // scale (8 - zero)
  };
};

template <bool I8, int G, int MT, int NT, int WK, int KC>
__global__ __launch_bounds__(W4_NT) void k_w4(W4Args a) {
  using S = W4Shape<I8, G, MT, NT, WK, KC>;
  __shared__ typename S::Buf buf[2];
  const int t = threadIdx.x, lane = lane_id(), wave = wave_id();
  const int c16 = lane & 15, q4 = lane >> 4;
  // The row blocks of one column block follow each other on one XCD (workgroups go round the 8 XCDs), which
  // then reads its weights once.
  const int nb = a.n_blocks, mb = a.m_blocks;
  int bn, bm;
  {
    const int id = blockIdx.x, full = nb / 8 * 8 * mb;
    if (id < full) {
      const int r = id % (8 * mb);
      bn = id / (8 * mb) * 8 + (r & 7);
      bm = r >> 3;
    } else {
      bn = nb / 8 * 8 + (id - full) % (nb % 8);
      bm = (id - full) / (nb % 8);
    }
  }
  const int64_t n0 = (int64_t)bn * S::RN;
  const int b0 = bm * S::ROWS;
  const int rows = min(S::ROWS, a.B - b0);
  const int rn = (int)min((int64_t)S::RN, a.N - n0);
  const int wn = WK == 1 ? wave * NT * 16 : 0;  // the wave's first weight row in the block
  const int wk = WK == 1 ? 0 : wave;
  const int row_bytes = a.K / 2, groups = a.K / G;

  const uint8_t* wrow[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) wrow[j] = a.q + (n0 + min(wn + j * 16 + c16, rn - 1)) * a.ldq;

  // staging: unit i of this thread is 16 bytes of one row; a group of columns lies in GL adjacent lanes
  constexpr int UPR = KC * S::ES / 16;          // units per row
  constexpr int GL = G * S::ES / 16;
  u32x4 xr[S::XPT];
  float sr[S::SPT];
  int zr[S::SPT];
  auto load_x = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < S::XPT; ++i) {
      const int u = t + i * W4_NT, r = u / UPR, k = k0 + (u % UPR) * (16 / S::ES);
      xr[i] = u32x4{0, 0, 0, 0};
      if (r < rows && k < a.K)
        xr[i] = *reinterpret_cast<const u32x4u*>(a.x + ((int64_t)(b0 + r) * a.ldx + k) * S::ES);
    }
  };
  auto load_s = [&](int k0) __attribute__((always_inline)) {
    const int g0 = k0 / G;
#pragma unroll
    for (int i = 0; i < S::SPT; ++i) {
      const int u = t + i * W4_NT, r = u / S::NG, g = g0 + u % S::NG;
      sr[i] = 0.0f;
      zr[i] = 8;
      if (r < rn && g < groups) {
        const int64_t at = (n0 + r) * a.lds + g;
        sr[i] = a.scale_bf16 ? BF16T::load1(a.scales, at) : F32T::load1(a.scales, at);
        if (a.zeros) zr[i] = a.zeros[(n0 + r) * a.ldz + g];
      }
    }
  };
  auto put = [&](typename S::Buf& b) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < S::XPT; ++i) {
      const int u = t + i * W4_NT, r = u / UPR, c = u % UPR;
      const u32x4 v = xr[i];
      u32x4 p;
      float sum;
      if constexpr (I8) {
        int s = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_sdot4((int)v[e], 0x01010101, s, false);
        s = (int)group_sum<GL>((uint32_t)s, [](uint32_t x, uint32_t y) { return x + y; });
        sum = (float)s;
        // columns 0 2 4 6 | 1 3 5 7 of each eight
        p[0] = __builtin_amdgcn_perm(v[1], v[0], 0x06040200u);
        p[1] = __builtin_amdgcn_perm(v[1], v[0], 0x07050301u);
        p[2] = __builtin_amdgcn_perm(v[3], v[2], 0x06040200u);
        p[3] = __builtin_amdgcn_perm(v[3], v[2], 0x07050301u);
      } else {
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s += __uint_as_float(v[e] << 16);
          s += __uint_as_float(v[e] & 0xffff0000u);
        }
        sum = __uint_as_float(group_sum<GL>(__float_as_uint(s), [](uint32_t x, uint32_t y) {
          return __float_as_uint(__uint_as_float(x) + __uint_as_float(y));
        }));
        // columns 0 4 | 1 5 | 2 6 | 3 7
        p[0] = __builtin_amdgcn_perm(v[2], v[0], 0x05040100u);
        p[1] = __builtin_amdgcn_perm(v[2], v[0], 0x07060302u);
        p[2] = __builtin_amdgcn_perm(v[3], v[1], 0x05040100u);
        p[3] = __builtin_amdgcn_perm(v[3], v[1], 0x07060302u);
      }
      if (r < rows) {
        *reinterpret_cast<u32x4*>(b.x + r * S::XST + c * 16) = p;
        if ((lane & (GL - 1)) == 0) b.sum[c / GL][r] = sum;
      }
    }
#pragma unroll
    for (int i = 0; i < S::SPT; ++i) {
      const int u = t + i * W4_NT, r = u / S::NG, g = u % S::NG;
      if (S::RN * S::NG % W4_NT == 0 || r < S::RN) {
        b.scale[g][r] = I8 ? sr[i] : 16.0f * sr[i];
        if (a.zeros) b.off[g][r] = sr[i] * (float)(8 - zr[i]);
      }
    }
  };
  auto load_w = [&](u32x4 (&w)[NT][S::KS], int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < S::KS; ++s) {
      const int at = min((k0 + (s * WK + wk) * 128) / 2 + q4 * 16, row_bytes - 16);
#pragma unroll
      for (int j = 0; j < NT; ++j) w[j][s] = *reinterpret_cast<const u32x4u*>(wrow[j] + at);
    }
  };

  f32x4 total[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < NT; ++j) total[m][j] = f32x4{0, 0, 0, 0};

  // Columns of step s (128) of the chunk: the operands of its instructions are NI sets; set i lies in group
  // i CH / ... of the step.  Where a group is 64 or 32 columns, the lanes of a load hold different groups, and
  // swaps between them put each group's columns into the same registers.
  constexpr int NI = I8 ? (G == 32 ? 4 : 2) : 4;  // instructions per 128 columns
  constexpr int GS = 128 / G;                     // groups per 128 columns
  auto multiply = [&](u32x4 (&w)[NT][S::KS], typename S::Buf& b, int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < S::KS; ++s) {
      const int ks = s * WK + wk;  // the step in the chunk
      if (k0 + ks * 128 >= a.K) break;
      u32x4 xa[MT][4];  // the step's columns of x, in the order of the weights below
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const unsigned char* xrow = b.x + (m * 16 + c16) * S::XST + ks * 128 * S::ES;
#pragma unroll
        for (int i = 0; i < (I8 ? 2 : 4); ++i) {
          int k;  // first of the 8 (bf16) or 16 (8 bits) columns
          if constexpr (!I8) {
            if constexpr (G == 128) k = q4 * 32 + i * 8;
            else if constexpr (G == 64) k = (i >> 1) * 64 + (q4 & 1) * 32 + (i & 1) * 16 + (q4 >> 1) * 8;
            else k = i * 32 + q4 * 8;
            xa[m][i] = *reinterpret_cast<const u32x4*>(xrow + k * 2);
          } else if constexpr (G == 128) {
            xa[m][i] = *reinterpret_cast<const u32x4*>(xrow + q4 * 32 + i * 16);
          } else if constexpr (G == 64) {
            xa[m][i] = *reinterpret_cast<const u32x4*>(xrow + i * 64 + (q4 & 1) * 32 + (q4 >> 1) * 16);
          } else {  // two groups of 32: eight columns of each
            const uint2 lo = *reinterpret_cast<const uint2*>(xrow + (2 * i) * 32 + q4 * 8);
            const uint2 hi = *reinterpret_cast<const uint2*>(xrow + (2 * i + 1) * 32 + q4 * 8);
            xa[m][i] = u32x4{lo.x, lo.y, hi.x, hi.y};
          }
        }
      }
      f32x4 sums[MT][GS];
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int g = 0; g < GS; ++g)
          sums[m][g] = *reinterpret_cast<const f32x4*>(&b.sum[ks * GS + g][m * 16 + q4 * 4]);
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        uint32_t d0 = w[j][s][0], d1 = w[j][s][1], d2 = w[j][s][2], d3 = w[j][s][3];
        if constexpr (G == 64 && !I8) {
          swap32(d0, d1);  // d0: group 0 (columns 0-7 and 8-15 of the two lanes), d1: group 1
          swap32(d2, d3);
          const uint32_t e = d1;
          d1 = d2;  // d0, d1: group 0; d2, d3: group 1
          d2 = e;
        } else if constexpr (G == 64) {
          swap32(d0, d2);  // (d0, d1): group 0, (d2, d3): group 1
          swap32(d1, d3);
        } else if constexpr (G == 32) {  // d[i]: group i
          swap32(d0, d2);
          swap32(d1, d3);
          swap16(d0, d1);
          swap16(d2, d3);
        }
        const uint32_t d[4] = {d0, d1, d2, d3};
        u32x4 wb[NI];
        if constexpr (!I8) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            wb[i][0] = ((d[i] << 3) & 0x00780078u) | 0x3f803f80u;
            wb[i][1] = ((d[i] >> 1) & 0x00780078u) | 0x3f803f80u;
            wb[i][2] = ((d[i] >> 5) & 0x00780078u) | 0x3f803f80u;
            wb[i][3] = ((d[i] >> 9) & 0x00780078u) | 0x3f803f80u;
          }
        } else if constexpr (G != 32) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            wb[i] = u32x4{d[2 * i] & 0x0f0f0f0fu, (d[2 * i] >> 4) & 0x0f0f0f0fu, d[2 * i + 1] & 0x0f0f0f0fu,
                          (d[2 * i + 1] >> 4) & 0x0f0f0f0fu};
        }
#pragma unroll
        for (int g = 0; g < GS; ++g) {
          const float sc = b.scale[ks * GS + g][wn + j * 16 + c16];
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            f32x4 r;
            if constexpr (I8) {
              i32x4 c;
#pragma unroll
              for (int e = 0; e < 4; ++e) c[e] = (int)(-8.0f * sums[m][g][e]);
              if constexpr (G == 32) {
                const u32x4 x4 = xa[m][g >> 1];
                const uint64_t xx = (g & 1) ? ((uint64_t)x4[3] << 32 | x4[2]) : ((uint64_t)x4[1] << 32 | x4[0]);
                const uint64_t ww = (uint64_t)((d[g] >> 4) & 0x0f0f0f0fu) << 32 | (d[g] & 0x0f0f0f0fu);
                c = __builtin_amdgcn_mfma_i32_16x16x32_i8((long)xx, (long)ww, c, 0, 0, 0);
              } else {
#pragma unroll
                for (int i = 0; i < 2 / GS; ++i)
                  c = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, xa[m][g * (2 / GS) + i]),
                                                            __builtin_bit_cast(i32x4, wb[g * (2 / GS) + i]), c, 0, 0, 0);
              }
#pragma unroll
              for (int e = 0; e < 4; ++e) r[e] = (float)c[e];
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) r[e] = -1.5f * sums[m][g][e];
#pragma unroll
              for (int i = 0; i < 4 / GS; ++i)
                r = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, xa[m][g * (4 / GS) + i]),
                                                            __builtin_bit_cast(bf16x8, wb[g * (4 / GS) + i]), r, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) total[m][j][e] = fmaf(r[e], sc, total[m][j][e]);
          }
          if (a.zeros) {
            const float of = b.off[ks * GS + g][wn + j * 16 + c16];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
              for (int e = 0; e < 4; ++e) total[m][j][e] = fmaf(sums[m][g][e], of, total[m][j][e]);
          }
        }
      }
    }
  };

  u32x4 wa[NT][S::KS], wb[NT][S::KS];
  load_x(0);
  load_s(0);
  load_w(wa, 0);
  put(buf[0]);
  // one chunk: the next one's loads go out, this one is multiplied, the next one's x goes to LDS
  auto chunk = [&](int k0, u32x4 (&cur)[NT][S::KS], u32x4 (&nxt)[NT][S::KS], int at) __attribute__((always_inline)) {
    const bool more = k0 + KC < a.K;
    if (more) {
      load_x(k0 + KC);
      load_s(k0 + KC);
      load_w(nxt, k0 + KC);
    }
    __syncthreads();
    multiply(cur, buf[at], k0);
    if (more) put(buf[at ^ 1]);
  };
  for (int k0 = 0; k0 < a.K; k0 += 2 * KC) {
    chunk(k0, wa, wb, 0);
    if (k0 + KC < a.K) chunk(k0 + KC, wb, wa, 1);
  }

  if constexpr (WK > 1) {  // join the waves' shares: wave 0 adds the others' in order
    static_assert(sizeof(f32x4) * 64 * MT * NT * (WK - 1) <= sizeof(buf), "the shares fit the staging buffers");
    f32x4* part = reinterpret_cast<f32x4*>(&buf[0]);
    __syncthreads();
    if (wave) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < NT; ++j) part[(((wave - 1) * MT + m) * NT + j) * 64 + lane] = total[m][j];
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 0; w < WK - 1; ++w)
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < NT; ++j) total[m][j] += part[((w * MT + m) * NT + j) * 64 + lane];
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int b = m * 16 + q4 * 4 + e;
      if (b < rows) {
        const float xs = I8 ? a.x_scale[b0 + b] : 1.0f;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const int n = wn + j * 16 + c16;
          if (n < rn) {
            const float v = I8 ? total[m][j][e] * xs : total[m][j][e];
            const int64_t at = (int64_t)(b0 + b) * a.ldo + n0 + n;
            if (a.out_bf16) store1<BF16T>(a.out, at, v);
            else store1<F32T>(a.out, at, v);
          }
        }
      }
    }
  }
}

template <bool I8, int G, int MT, int NT, int WK, int KC>
hipError_t launch(W4Args& a, hipStream_t stream) {
  using S = W4Shape<I8, G, MT, NT, WK, KC>;
  const int64_t nb = (a.N + S::RN - 1) / S::RN, mb = (a.B + S::ROWS - 1) / S::ROWS;
  if (nb * mb >= ((int64_t)1 << 31)) return hipErrorInvalidConfiguration;
  a.n_blocks = (int32_t)nb;
  a.m_blocks = (int32_t)mb;
  hipLaunchKernelGGL((k_w4<I8, G, MT, NT, WK, KC>), dim3((unsigned)(nb * mb)), dim3(W4_NT), 0, stream, a);
  return hipGetLastError();
}

// Tiles by the number of rows: as many 16-row operands as the rows fill, up to four, so that a weight is
// unpacked once for up to 64 rows.
template <bool I8, int G>
hipError_t launch_rows(W4Args& a, hipStream_t stream) {
  if (a.B <= 16) {
    if (a.N < 16384) return launch<I8, G, 1, 1, 4, 1024>(a, stream);
    return launch<I8, G, 1, 2, 1, 512>(a, stream);
  }
  if (a.B <= 32) return launch<I8, G, 2, 2, 1, 256>(a, stream);
  return launch<I8, G, 4, 4, 1, 128>(a, stream);
}

}  // namespace

extern "C" {

albireo_status_t albireo_matmul_w4(const void* x, albireo_rows_t x_type, int64_t B, int64_t ldx,
                                   const float* x_scale, const albireo_w4_t* weight, void* out,
                                   albireo_dtype_t out_dtype, int64_t ldo, hipStream_t stream) {
  if (x_type != ALBIREO_ROWS_BF16 && x_type != ALBIREO_ROWS_I8) return ALBIREO_E_INVALID;
  if (out_dtype != ALBIREO_F32 && out_dtype != ALBIREO_BF16) return ALBIREO_E_INVALID;
  if (!weight) return ALBIREO_E_INVALID;
  const albireo_w4_t& w = *weight;
  if (w.scale_dtype != ALBIREO_F32 && w.scale_dtype != ALBIREO_BF16) return ALBIREO_E_INVALID;
  if (w.group != 32 && w.group != 64 && w.group != 128) return ALBIREO_E_INVALID;
  if (B < 0 || w.N < 0 || w.K <= 0 || w.K % w.group || ldx < w.K || ldo < w.N) return ALBIREO_E_INVALID;
  if (w.ldq < w.K / 2 || w.lds < w.K / w.group || (w.zeros && w.ldz < w.K / w.group)) return ALBIREO_E_INVALID;
  const bool i8 = x_type == ALBIREO_ROWS_I8;
  if (!i8 && x_scale) return ALBIREO_E_INVALID;
  if (B > 65535 || w.N >= ((int64_t)1 << 31) - 1024 || w.K >= ((int64_t)1 << 24)) return ALBIREO_E_UNSUPPORTED;
  const auto off = [](const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; };
  if (off(x, i8 ? 1 : 2) || off(x_scale, 4) || off(out, out_dtype == ALBIREO_BF16 ? 2 : 4) ||
      off(w.scales, w.scale_dtype == ALBIREO_BF16 ? 2 : 4))
    return ALBIREO_E_INVALID;
  if (B == 0 || w.N == 0) return ALBIREO_OK;
  if (!x || !out || !w.q || !w.scales || (i8 && !x_scale)) return ALBIREO_E_INVALID;

  W4Args a;
  a.x = static_cast<const unsigned char*>(x);
  a.x_scale = x_scale;
  a.q = w.q;
  a.scales = static_cast<const unsigned char*>(w.scales);
  a.zeros = w.zeros;
  a.out = static_cast<unsigned char*>(out);
  a.ldx = ldx, a.ldq = w.ldq, a.lds = w.lds, a.ldz = w.ldz, a.ldo = ldo;
  a.N = w.N;
  a.B = (int32_t)B, a.K = (int32_t)w.K;
  a.scale_bf16 = w.scale_dtype == ALBIREO_BF16;
  a.out_bf16 = out_dtype == ALBIREO_BF16;
  hipError_t e;
  if (i8) e = w.group == 128 ? launch_rows<true, 128>(a, stream)
            : w.group == 64  ? launch_rows<true, 64>(a, stream) : launch_rows<true, 32>(a, stream);
  else e = w.group == 128 ? launch_rows<false, 128>(a, stream)
         : w.group == 64  ? launch_rows<false, 64>(a, stream) : launch_rows<false, 32>(a, stream);
  return e == hipSuccess ? ALBIREO_OK : ALBIREO_E_LAUNCH;
}

}  // extern "C"
