// adjust.hip -- albireo_adjust_logits: biases, penalties and grammar masks on the logits.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>
#include <string.h>

#include <utility>

#include "albireo_decode.h"
#include "checks.h"

namespace {

#include "common.h"
#include "rows.h"

constexpr int ADJ_NT = 256;
constexpr int ADJ_TILE = 8192;

struct AdjArgs {
  const unsigned char* logits;
  unsigned char* out;
  uint32_t* flags;
  int64_t V, ld, ldo;
  DevParams prm;
  const int64_t* prompt_offsets;
  const int32_t* prompt_ids;
  int64_t prompt_len;
  const int32_t* st_ids;
  const uint32_t* st_counts;
  const int32_t* st_len;
  const uint32_t* st_flags;
  int32_t st_cap;
  const int64_t* bias_offsets;
  const int32_t* bias_ids;
  const float* bias_values;
  int64_t bias_len;
  const uint32_t* mask;
  int64_t mask_rows, mask_ld;
  const int32_t* mask_index;
};

// the range of a row's CSR list; a malformed one is empty
__device__ __forceinline__ bool csr_range(const int64_t* offsets, int64_t row, int64_t len, int64_t& lo, int64_t& hi) {
  lo = hi = 0;
  if (!offsets) return true;
  lo = sload(offsets + row);
  hi = sload(offsets + row + 1);
  if (lo >= 0 && hi >= lo && hi <= len) return true;
  lo = hi = 0;
  return false;
}

// One tile of one row per workgroup.
template <class DT, class OT>
__global__ __launch_bounds__(ADJ_NT) void k_adjust(AdjArgs a) {
  __shared__ uint32_t word[ADJ_TILE];
  __shared__ float val[ADJ_TILE];
  const int t = threadIdx.x;
  const int64_t row = blockIdx.y;
  const int64_t t0 = (int64_t)blockIdx.x * ADJ_TILE, t1 = min(a.V, t0 + ADJ_TILE);
  const unsigned char* xr = a.logits + row * a.ld * DT::ES;
  unsigned char* orow = a.out + row * a.ldo * OT::ES;
  const DevParams& q = a.prm;
  uint32_t fl = 0;
  float rep = sload(q.rep ? q.rep + row : &kParamDefaults[3]);
  float freq = sload(q.freq ? q.freq + row : &kParamDefaults[4]);
  float pres = sload(q.pres ? q.pres + row : &kParamDefaults[5]);
  if (!(rep > 0.0f) || isinf(rep)) rep = 1.0f, fl |= FLAG_BAD_PARAM;
  if (!isfinite(freq)) freq = 0.0f, fl |= FLAG_BAD_PARAM;
  if (!isfinite(pres)) pres = 0.0f, fl |= FLAG_BAD_PARAM;
  int64_t lo, hi, plo, phi, blo, bhi;
  if (!csr_range(q.hist_offsets, row, q.hist_len, lo, hi)) fl |= FLAG_BAD_PARAM;
  if (!csr_range(a.prompt_offsets, row, a.prompt_len, plo, phi)) fl |= FLAG_BAD_PARAM;
  if (!csr_range(a.bias_offsets, row, a.bias_len, blo, bhi)) fl |= FLAG_BAD_PARAM;
  int sn = 0;
  if (a.st_len) {
    sn = sload(a.st_len + row);
    sn = sn < 0 ? 0 : (sn > a.st_cap ? a.st_cap : sn);
  }
  const uint32_t* mrow = nullptr;
  if (a.mask) {
    int64_t m = row;
    if (a.mask_index) m = a.mask_index[row];
    if (m >= a.mask_rows) fl |= FLAG_BAD_PARAM;
    else if (m >= 0) mrow = a.mask + m * a.mask_ld;
  }
  for (int i = t; i < (int)(t1 - t0); i += ADJ_NT) {
    val[i] = DT::load1(xr, t0 + i);
    word[i] = 0;
  }
  __syncthreads();
  for (int64_t e = blo + t; e < bhi; e += ADJ_NT) {  // the last entry of an id
    const int32_t id = a.bias_ids[e];
    if (id < 0 || id >= a.V) fl |= FLAG_BAD_INPUT;
    else if (isnan(a.bias_values[e])) fl |= FLAG_BAD_PARAM;
    if (id >= t0 && id < t1) atomicMax(&word[id - t0], (uint32_t)(e - blo) + 1u);
  }
  __syncthreads();
  for (int i = t; i < (int)(t1 - t0); i += ADJ_NT) {
    if (word[i]) {
      const float b = a.bias_values[blo + word[i] - 1];
      if (!isnan(b)) val[i] = __fadd_rn(val[i], b);
    }
    word[i] = 0;
  }
  __syncthreads();
  for (int64_t e = lo + t; e < hi; e += ADJ_NT) {
    const int32_t id = q.hist_ids[e];
    if (id < 0 || id >= a.V) fl |= FLAG_BAD_INPUT;
    if (id >= t0 && id < t1) atomicAdd(&word[id - t0], 1u);
  }
  for (int64_t e = plo + t; e < phi; e += ADJ_NT) {
    const int32_t id = a.prompt_ids[e];
    if (id < 0 || id >= a.V) fl |= FLAG_BAD_INPUT;
    if (id >= t0 && id < t1) atomicOr(&word[id - t0], 0x80000000u);
  }
  for (int e = t; e < sn; e += ADJ_NT) {
    const int32_t id = a.st_ids[row * a.st_cap + e];
    if (id < 0 || id >= a.V) fl |= FLAG_BAD_INPUT;
    if (id >= t0 && id < t1) word[id - t0] = a.st_counts[row * a.st_cap + e];
  }
  __syncthreads();
  for (int i = t; i < (int)(t1 - t0); i += ADJ_NT) {
    const int64_t v = t0 + i;
    float x = val[i];
    if (word[i]) x = penalise_cv(x, word[i], rep, freq, pres);
    if (mrow && !((mrow[v >> 5] >> (v & 31)) & 1u)) x = -INFINITY;
    store1<OT>(orow, v, x);
  }
  if (a.flags && blockIdx.x == 0) {
    const uint32_t f1 = __syncthreads_or(fl & FLAG_BAD_INPUT) ? FLAG_BAD_INPUT : 0u;
    const uint32_t f2 = __syncthreads_or(fl & FLAG_BAD_PARAM) ? FLAG_BAD_PARAM : 0u;
    if (t == 0) a.flags[row] = f1 | f2 | (a.st_flags ? a.st_flags[row] : 0u);
  }
}

}  // namespace

extern "C" {

albireo_status_t albireo_adjust_logits(const void* logits, albireo_dtype_t dtype, int64_t B, int64_t V, int64_t ld,
                                       const albireo_params_t* params, const albireo_constraints_t* constraints,
                                       void* out, albireo_dtype_t out_dtype, int64_t ldo, uint32_t* out_flags,
                                       hipStream_t stream) {
  albireo_status_t st = check_common(logits, dtype, B, V, ld, params);
  if (st != ALBIREO_OK) return st;
  if ((out_dtype != ALBIREO_F32 && out_dtype != ALBIREO_BF16) || ldo < V) return ALBIREO_E_INVALID;
  if (reinterpret_cast<uintptr_t>(out) % (out_dtype == ALBIREO_BF16 ? 2 : 4)) return ALBIREO_E_INVALID;
  if (reinterpret_cast<uintptr_t>(out_flags) % 4) return ALBIREO_E_INVALID;
  if (constraints && constraints->bias_offsets) {
    if (constraints->bias_len < 0 || constraints->bias_len >= ((int64_t)1 << 32) - 1) return ALBIREO_E_INVALID;
    if (constraints->bias_len > 0 && (!constraints->bias_ids || !constraints->bias_values)) return ALBIREO_E_INVALID;
  }
  if (constraints && constraints->mask) {
    if (constraints->mask_rows < 0 || constraints->mask_ld < (V + 31) / 32) return ALBIREO_E_INVALID;
    if (!constraints->mask_index && constraints->mask_rows < B) return ALBIREO_E_INVALID;
    if (reinterpret_cast<uintptr_t>(constraints->mask) % 4) return ALBIREO_E_INVALID;
  }
  if (B == 0) return ALBIREO_OK;
  if (!out) return ALBIREO_E_INVALID;
  if (out == logits && (out_dtype != dtype || ldo != ld)) return ALBIREO_E_INVALID;
  if (B > 65535) return ALBIREO_E_UNSUPPORTED;

  AdjArgs a;
  memset(&a, 0, sizeof a);
  a.logits = static_cast<const unsigned char*>(logits);
  a.out = static_cast<unsigned char*>(out);
  a.flags = out_flags;
  a.V = V, a.ld = ld, a.ldo = ldo;
  if (params) {
    a.prm.rep = params->repetition_penalty;
    a.prm.freq = params->frequency_penalty;
    a.prm.pres = params->presence_penalty;
    a.prm.hist_offsets = params->hist_offsets;
    a.prm.hist_ids = params->hist_ids;
    a.prm.hist_len = params->hist_len;
    a.prompt_offsets = params->prompt_offsets;
    a.prompt_ids = params->prompt_ids;
    a.prompt_len = params->prompt_len;
    if (params->state) {
      a.st_ids = params->state->ids;
      a.st_counts = params->state->counts;
      a.st_len = params->state->len;
      a.st_flags = params->state->flags;
      a.st_cap = params->state->cap;
    }
  }
  if (constraints) {
    a.bias_offsets = constraints->bias_offsets;
    a.bias_ids = constraints->bias_ids;
    a.bias_values = constraints->bias_values;
    a.bias_len = constraints->bias_len;
    a.mask = constraints->mask;
    a.mask_rows = constraints->mask_rows;
    a.mask_ld = constraints->mask_ld;
    a.mask_index = constraints->mask_index;
  }
  const dim3 grid((unsigned)((V + ADJ_TILE - 1) / ADJ_TILE), (unsigned)B), nt(ADJ_NT);
  if (dtype == ALBIREO_BF16) {
    if (out_dtype == ALBIREO_BF16) hipLaunchKernelGGL((k_adjust<BF16T, BF16T>), grid, nt, 0, stream, a);
    else hipLaunchKernelGGL((k_adjust<BF16T, F32T>), grid, nt, 0, stream, a);
  } else {
    if (out_dtype == ALBIREO_BF16) hipLaunchKernelGGL((k_adjust<F32T, BF16T>), grid, nt, 0, stream, a);
    else hipLaunchKernelGGL((k_adjust<F32T, F32T>), grid, nt, 0, stream, a);
  }
  return hipGetLastError() == hipSuccess ? ALBIREO_OK : ALBIREO_E_LAUNCH;
}

}  // extern "C"
