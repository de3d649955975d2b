// norm.hip -- albireo_rms_norm: residual addition and root-mean-square norm of hidden states, in the
// inputs' type and / or in 8 bits with a scale per row.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>
#include <string.h>

#include <utility>

#include "albireo_decode.h"

namespace {

#include "common.h"
#include "rows.h"

struct NormArgs {
  const unsigned char* x;
  const unsigned char* residual;
  const unsigned char* weight;
  unsigned char* out_residual;
  unsigned char* out;
  int8_t* out_q;
  float* out_scale;
  int64_t ldx, ldr, ldro, ldo, ldq;
  int32_t D;
  float eps;
};

constexpr int NORM_NT = 256;

// One workgroup per row, three passes over it.
template <class DT, class WT>
__global__ __launch_bounds__(NORM_NT) void k_norm(NormArgs a) {
  __shared__ float h[ALBIREO_MAX_NORM_WIDTH];
  __shared__ double red[NORM_NT / 64];
  __shared__ float redm[NORM_NT / 64];
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x;
  const unsigned char* xr = a.x + row * a.ldx * DT::ES;
  const unsigned char* rr = a.residual ? a.residual + row * a.ldr * DT::ES : nullptr;
  double ss = 0.0;
  for (int i = t; i < a.D; i += NORM_NT) {
    float v = DT::load1(xr, i);
    if (rr) v += DT::load1(rr, i);
    h[i] = v;
    ss += (double)v * (double)v;
  }
  for (int d = 32; d; d >>= 1) ss += __shfl_xor(ss, d);
  if (lane_id() == 0) red[wave_id()] = ss;
  __syncthreads();
  ss = ((red[0] + red[1]) + red[2]) + red[3];
  const float rstd = (float)(1.0 / sqrt(ss / a.D + (double)a.eps));
  float amax = 0.0f;
  bool bad = !isfinite(ss);
  for (int i = t; i < a.D; i += NORM_NT) {
    const float w = a.weight ? WT::load1(a.weight, i) : 1.0f;
    const float y = h[i] * rstd * w;
    if (a.out_residual) store1<DT>(a.out_residual + row * a.ldro * DT::ES, i, h[i]);
    if (a.out) store1<DT>(a.out + row * a.ldo * DT::ES, i, y);
    bad |= !isfinite(y);
    amax = fmaxf(amax, fabsf(y));
    h[i] = y;
  }
  if (!a.out_q) return;
  amax = wave_max(amax);
  if (lane_id() == 0) redm[wave_id()] = amax;
  bad = __syncthreads_or(bad);
  amax = fmaxf(fmaxf(redm[0], redm[1]), fmaxf(redm[2], redm[3]));
  const bool zero = bad || amax < 0x1p-120f;
  const float inv = zero ? 0.0f : 127.0f / amax;
  for (int i = t; i < a.D; i += NORM_NT) a.out_q[row * a.ldq + i] = zero ? 0 : (int8_t)(int)rintf(h[i] * inv);
  if (t == 0) a.out_scale[row] = bad ? __uint_as_float(0x7fc00000u) : (zero ? 0.0f : amax / 127.0f);
}

}  // namespace

extern "C" {

albireo_status_t albireo_rms_norm(const void* x, albireo_dtype_t dtype, int64_t T, int64_t D, int64_t ldx,
                                  const void* residual, int64_t ldr, const void* weight,
                                  albireo_dtype_t weight_dtype, float eps, void* out_residual, int64_t ldro,
                                  void* out, int64_t ldo, int8_t* out_q, int64_t ldq, float* out_scale,
                                  hipStream_t stream) {
  if (dtype != ALBIREO_F32 && dtype != ALBIREO_BF16) return ALBIREO_E_INVALID;
  if (weight && weight_dtype != ALBIREO_F32 && weight_dtype != ALBIREO_BF16) return ALBIREO_E_INVALID;
  if (T < 0 || D <= 0 || ldx < D) return ALBIREO_E_INVALID;
  if (!(eps > 0.0f) || isinf(eps)) return ALBIREO_E_INVALID;
  if (residual && ldr < D) return ALBIREO_E_INVALID;
  if (out_residual && ldro < D) return ALBIREO_E_INVALID;
  if (out && ldo < D) return ALBIREO_E_INVALID;
  if ((out_q != nullptr) != (out_scale != nullptr)) return ALBIREO_E_INVALID;
  if (out_q && ldq < D) return ALBIREO_E_INVALID;
  if (D > ALBIREO_MAX_NORM_WIDTH || T >= ((int64_t)1 << 31)) return ALBIREO_E_UNSUPPORTED;
  const uintptr_t es = dtype == ALBIREO_BF16 ? 2 : 4, ws = weight_dtype == ALBIREO_BF16 ? 2 : 4;
  const auto off = [](const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; };
  if (off(x, es) || off(residual, es) || off(out_residual, es) || off(out, es) || off(out_scale, 4)) return ALBIREO_E_INVALID;
  if (weight && off(weight, ws)) return ALBIREO_E_INVALID;
  // an output in place of an input needs its stride, and two outputs cannot share an array
  if (out && out == out_residual) return ALBIREO_E_INVALID;
  for (const auto& o : {std::make_pair((const void*)out, ldo), std::make_pair((const void*)out_residual, ldro)}) {
    if (!o.first) continue;
    if (o.first == x && o.second != ldx) return ALBIREO_E_INVALID;
    if (o.first == residual && o.second != ldr) return ALBIREO_E_INVALID;
  }
  if (T == 0) return ALBIREO_OK;
  if (!x || (!out_residual && !out && !out_q)) return ALBIREO_E_INVALID;

  NormArgs a;
  a.x = static_cast<const unsigned char*>(x);
  a.residual = static_cast<const unsigned char*>(residual);
  a.weight = static_cast<const unsigned char*>(weight);
  a.out_residual = static_cast<unsigned char*>(out_residual);
  a.out = static_cast<unsigned char*>(out);
  a.out_q = out_q;
  a.out_scale = out_scale;
  a.ldx = ldx, a.ldr = ldr, a.ldro = ldro, a.ldo = ldo, a.ldq = ldq;
  a.D = (int32_t)D;
  a.eps = eps;
  const bool wb = weight && weight_dtype == ALBIREO_BF16;
  const dim3 grid((unsigned)T);
  if (dtype == ALBIREO_BF16) {
    if (wb) hipLaunchKernelGGL((k_norm<BF16T, BF16T>), grid, dim3(NORM_NT), 0, stream, a);
    else hipLaunchKernelGGL((k_norm<BF16T, F32T>), grid, dim3(NORM_NT), 0, stream, a);
  } else {
    if (wb) hipLaunchKernelGGL((k_norm<F32T, BF16T>), grid, dim3(NORM_NT), 0, stream, a);
    else hipLaunchKernelGGL((k_norm<F32T, F32T>), grid, dim3(NORM_NT), 0, stream, a);
  }
  return hipGetLastError() == hipSuccess ? ALBIREO_OK : ALBIREO_E_LAUNCH;
}

}  // extern "C"
