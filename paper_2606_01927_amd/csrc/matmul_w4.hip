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
  int32_t B, K, group;
};

// One wave per output.
template <bool I8, class ST, class OT>
__global__ __launch_bounds__(256) void k_w4(W4Args a) {
  const int64_t n = (int64_t)blockIdx.x * 4 + wave_id();
  const int64_t b = blockIdx.y;
  if (n >= a.N) return;
  const uint8_t* qr = a.q + n * a.ldq;
  const unsigned char* xr = a.x + b * a.ldx * (I8 ? 1 : 2);
  float acc = 0.0f;
  for (int k0 = lane_id() * 8; k0 < a.K; k0 += 512) {
    const int g = k0 / a.group;
    const float s = ST::load1(a.scales + n * a.lds * ST::ES, g);
    const int z = a.zeros ? a.zeros[n * a.ldz + g] : 8;
    float p = 0.0f;
    for (int e = 0; e < 8; ++e) {
      const int w = (qr[(k0 + e) >> 1] >> (4 * (e & 1))) & 15;
      float x;
      if constexpr (I8) x = (float)reinterpret_cast<const int8_t*>(xr)[k0 + e];
      else x = BF16T::load1(xr, k0 + e);
      p = fmaf(x, (float)(w - z), p);
    }
    acc = fmaf(p, s, acc);
  }
  acc = wave_sum(acc);
  if (I8) acc *= a.x_scale[b];
  if (lane_id() == 0) {
    store1<OT>(a.out + b * a.ldo * OT::ES, n, acc);
  }
}

template <bool I8, class ST>
void launch_out(const W4Args& a, albireo_dtype_t out_dtype, dim3 grid, hipStream_t stream) {
  if (out_dtype == ALBIREO_BF16) hipLaunchKernelGGL((k_w4<I8, ST, BF16T>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((k_w4<I8, ST, F32T>), grid, dim3(256), 0, stream, a);
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
  a.B = (int32_t)B, a.K = (int32_t)w.K, a.group = w.group;
  const dim3 grid((unsigned)((w.N + 3) / 4), (unsigned)B);
  if (i8) {
    if (w.scale_dtype == ALBIREO_BF16) launch_out<true, BF16T>(a, out_dtype, grid, stream);
    else launch_out<true, F32T>(a, out_dtype, grid, stream);
  } else {
    if (w.scale_dtype == ALBIREO_BF16) launch_out<false, BF16T>(a, out_dtype, grid, stream);
    else launch_out<false, F32T>(a, out_dtype, grid, stream);
  }
  return hipGetLastError() == hipSuccess ? ALBIREO_OK : ALBIREO_E_LAUNCH;
}

}  // extern "C"
