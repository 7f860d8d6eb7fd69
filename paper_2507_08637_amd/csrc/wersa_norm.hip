// Root-mean-square norm over the columns of a row, with the residual's addition before it:
//   r = x + residual (rounded to the tensors' type: the stream that the next layer adds to),  rstd = (mean(r^2) + eps)^-1/2,  y = r rstd weight
// and its derivative.  Sums in float32.  Everything here is bound by memory: a row is read once and stays in registers.
#include "wersa_rows.h"

namespace wersa {
namespace {

struct NormJob {
  const void *x, *residual;
  const float *weight;
  void *r, *y;
  float *rstd, *scales;
  int64_t rows, stride_x, stride_residual;
  int cols;
  float eps;
};

// LANES threads to a row, PIECES pieces of 16 bytes to a thread.  131072 rows of 2048 in bf16 with a residual: 365 us, 5.9 TB/s; to 8 bits 328 us, 5.7 TB/s (a copy: 5.7).
template <typename T, int LANES, int PIECES, bool EIGHT>
__global__ __launch_bounds__(256) void norm_kernel(NormJob a) {
  constexpr int E = 16 / sizeof(T);
  __shared__ float part[4];
  const int t = threadIdx.x % LANES;
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
  const bool ok = row < a.rows;   // (every thread stays for the sums)
  const T *x = (const T *)a.x + (ok ? row : 0) * a.stride_x;
  float v[PIECES][E];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) load_piece<T, E>(x, (t + LANES * p) * E, ok ? a.cols : 0, v[p]);
  if (a.residual) {
    const T *res = (const T *)a.residual + (ok ? row : 0) * a.stride_residual;
    T *r = (T *)a.r + (ok ? row : 0) * a.cols;
    float u[PIECES][E];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) load_piece<T, E>(res, (t + LANES * p) * E, ok ? a.cols : 0, u[p]);
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
#pragma unroll
      for (int i = 0; i < E; ++i) v[p][i] = rounded<T>(v[p][i] + u[p][i]);
      store_piece<T, E>(r, (t + LANES * p) * E, ok ? a.cols : 0, v[p]);
    }
  }
  float sum = 0.f;
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) s += v[p][i] * v[p][i];
    sum += s;
  }
  const float rstd = rsqrtf(row_sum<LANES>(sum, part) / (float)a.cols + a.eps);
  if (a.rstd && ok && t == 0) a.rstd[row] = rstd;
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    float w[E];
    load_weights(a.weight, (t + LANES * p) * E, a.cols, w);
#pragma unroll
    for (int i = 0; i < E; ++i) v[p][i] = v[p][i] * rstd * w[i];
  }
  if (!EIGHT) {
    T *y = (T *)a.y + (ok ? row : 0) * a.cols;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) store_piece<T, E>(y, (t + LANES * p) * E, ok ? a.cols : 0, v[p]);
    return;
  }
  // e4m3 (largest value 448) with one scale for the row; a row of zeros has scale 1
  uint32_t most = 0;
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int i = 0; i < E; ++i) most = max(most, __float_as_uint(v[p][i]) & 0x7fffffffu);
  const float top = __uint_as_float(row_most<LANES>(most, part));
  float inverse = top > 0.f ? 448.f / top : 1.f;
  if (top > 0.f && top < 0x1p-100f) {   // a row so small that 448 / top may leave float32: its values are raised first
    inverse = 448.f / (top * 0x1p64f);
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int i = 0; i < E; ++i) v[p][i] *= 0x1p64f;
  }
  if (ok && t == 0) a.scales[row] = top > 0.f ? top / 448.f : 1.f;
  unsigned char *y = (unsigned char *)a.y + (ok ? row : 0) * a.cols;
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    uint32_t bits[E / 4];
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      int b = __builtin_amdgcn_cvt_pk_fp8_f32(v[p][i] * inverse, v[p][i + 1] * inverse, 0, false);
      bits[i / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[p][i + 2] * inverse, v[p][i + 3] * inverse, b, true);
    }
    const int col = (t + LANES * p) * E;
    if (ok && col + E <= a.cols) {
      if (E == 8) *reinterpret_cast<u32x2_any *>(y + col) = u32x2{bits[0], bits[E / 4 - 1]};
      else *reinterpret_cast<u32_any *>(y + col) = bits[0];
    } else if (ok) {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (col + i < a.cols) y[col + i] = (unsigned char)(bits[i / 4] >> (8 * (i % 4)));
    }
  }
}

// Workgroups of the backward at most: three to a compute unit, two where a thread holds 32 columns (weights, sums and three tensors' values in registers).
// 131072 rows of 2048 in bf16: 413 us with 512, 433 with 768, 719 with three to a unit and registers in scratch; 128000 rows of 128 in float32: 44.4 with 768, 47.2 with 512.
constexpr int kBackGroups = 768;
__host__ __device__ constexpr int back_groups(int columns) { return columns >= 32 ? 512 : kBackGroups; }   // columns of a thread

struct NormBackJob {
  const void *r, *dy, *dr;
  const float *weight, *rstd;
  void *dx;
  float *partial;           // [workgroup][cols]: sums of dy xhat over its rows; null: not wanted
  int64_t rows, stride_r;
  int cols;
};

// dx = rstd (g - xhat mean(g xhat)) + dr with g = dy weight.  A workgroup takes rows from its index on, as many at a time as it holds, with the weights of its
// columns and their sums of dy xhat in registers throughout.  All that a row needs is requested before the first of it is used; it stays as it came, and is taken apart twice.
template <typename T, int LANES, int PIECES>
__global__ __launch_bounds__(256, back_groups(PIECES * 16 / sizeof(T)) / 256) void norm_back_kernel(NormBackJob a) {
  constexpr int E = 16 / sizeof(T), ROWS = 256 / LANES;
  __shared__ float part[4];
  __shared__ float sums[LANES == 256 ? 1 : 256 * 4];
  const int t = threadIdx.x % LANES;
  float w[PIECES][E], dw[PIECES][E];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    load_weights(a.weight, (t + LANES * p) * E, a.cols, w[p]);
#pragma unroll
    for (int i = 0; i < E; ++i) dw[p][i] = 0.f;
  }
  for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < a.rows; row0 += (int64_t)gridDim.x * ROWS) {
    const int64_t row = row0 + threadIdx.x / LANES, at = row < a.rows ? row : 0;
    const int cols = row < a.rows ? a.cols : 0;
    const T *r = (const T *)a.r + at * a.stride_r, *dy = (const T *)a.dy + at * a.cols, *dr = (const T *)a.dr + at * a.cols;
    u32x4 rr[PIECES], rd[PIECES], ru[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      rr[p] = load_raw(r, (t + LANES * p) * E, cols);
      rd[p] = load_raw(dy, (t + LANES * p) * E, cols);
    }
    if (a.dr) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) ru[p] = load_raw(dr, (t + LANES * p) * E, cols);
    }
    const float rstd = a.rstd[at];
    float dot = 0.f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      float v[E], g[E], s = 0.f;
      spread<T, E>(rr[p], v);
      spread<T, E>(rd[p], g);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        v[i] *= rstd;
        dw[p][i] += g[i] * v[i];
        s += g[i] * w[p][i] * v[i];
      }
      dot += s;
    }
    const float mean = row_sum<LANES>(dot, part) / (float)a.cols;
    T *dx = (T *)a.dx + at * a.cols;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      float v[E], g[E], u[E];
      spread<T, E>(rr[p], v);
      spread<T, E>(rd[p], g);
      if (a.dr) spread<T, E>(ru[p], u);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        g[i] = rstd * (g[i] * w[p][i] - v[i] * rstd * mean);
        if (a.dr) g[i] += u[i];
      }
      store_piece<T, E>(dx, (t + LANES * p) * E, cols, g);
    }
  }
  if (!a.partial) return;
  float *out = a.partial + (int64_t)blockIdx.x * a.cols;
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int i0 = 0; i0 < E; i0 += 4) {
      if (LANES < 256) {   // the rows of the workgroup
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[i * 256 + threadIdx.x] = dw[p][i0 + i];
        __syncthreads();
      }
      if (threadIdx.x < LANES) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float s = dw[p][i0 + i];
          if (LANES < 256) {
#pragma unroll
            for (int u = 1; u < ROWS; ++u) s += sums[i * 256 + u * LANES + threadIdx.x];
          }
          const int col = (t + LANES * p) * E + i0 + i;
          if (col < a.cols) out[col] = s;
        }
      }
    }
}

// Sum over the workgroups: 16 columns, 64 shares of the workgroups, all requests of a share at once.
__global__ __launch_bounds__(1024) void norm_reduce_kernel(const float *partial, int groups, int cols, float *dweight) {
  constexpr int SHARES = 64, EACH = kBackGroups / SHARES;
  __shared__ float part[SHARES][17];
  const int c = threadIdx.x % 16, s = threadIdx.x / 16, col = blockIdx.x * 16 + c;
  float v[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) v[i] = col < cols && s + SHARES * i < groups ? partial[(int64_t)(s + SHARES * i) * cols + col] : 0.f;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < EACH; ++i) sum += v[i];
  part[s][c] = sum;
#pragma unroll
  for (int d = SHARES / 2; d > 0; d /= 2) {
    __syncthreads();
    if (s < d) part[s][c] += part[s + d][c];
  }
  if (s == 0 && col < cols) dweight[col] = part[0][c];
}


wersa_status validate(const wersa_norm_desc *c) {
  if (!c) return WERSA_ERR_INVALID_ARG;
  if (c->rows < 0 || c->cols < 1 || !(c->eps >= 0.f)) return WERSA_ERR_INVALID_ARG;
  if (c->dtype != WERSA_F32 && c->dtype != WERSA_BF16) return WERSA_ERR_INVALID_ARG;
  if (c->rows > 1 && (c->stride_x < c->cols || c->stride_residual < c->cols)) return WERSA_ERR_INVALID_ARG;
  if (c->cols > 8192 || c->rows > ((int64_t)1 << 31)) return WERSA_ERR_UNSUPPORTED;
  return WERSA_OK;
}

wersa_status forward(const wersa_norm_desc &c, const NormJob &a, bool eight, hipStream_t st) {
  by_width(c.cols, c.dtype, [&](auto *type, auto lanes, auto pieces) {
    typedef typename std::remove_pointer<decltype(type)>::type T;
    constexpr int L = decltype(lanes)::value, P = decltype(pieces)::value;
    const dim3 grid = grid_of((c.rows + 256 / L - 1) / (256 / L));
    if (eight) WERSA_STAGE("wersa_rms_norm_eight_bit", st, (norm_kernel<T, L, P, true><<<grid, 256, 0, st>>>(a)));
    else WERSA_STAGE("wersa_rms_norm", st, (norm_kernel<T, L, P, false><<<grid, 256, 0, st>>>(a)));
  });
  return hipGetLastError() == hipSuccess ? WERSA_OK : WERSA_ERR_LAUNCH;
}

}  // namespace
}  // namespace wersa

using namespace wersa;

extern "C" {

wersa_status wersa_rms_norm_forward(const wersa_norm_desc *desc, const void *x, const void *residual, const float *weight, void *r, void *y,
                                    float *rstd, void *hip_stream) {
  const wersa_status vs = validate(desc);
  if (vs != WERSA_OK) return vs;
  if (desc->rows == 0) return WERSA_OK;
  if (!x || !y || (residual && !r)) return WERSA_ERR_INVALID_ARG;
  const NormJob a{x, residual, weight, r, y, rstd, nullptr, desc->rows, desc->stride_x, desc->stride_residual, desc->cols, desc->eps};
  return forward(*desc, a, false, (hipStream_t)hip_stream);
}

wersa_status wersa_rms_norm_eight_bit(const wersa_norm_desc *desc, const void *x, const void *residual, const float *weight, void *r, void *y,
                                      float *scales, void *hip_stream) {
  const wersa_status vs = validate(desc);
  if (vs != WERSA_OK) return vs;
  if (desc->rows == 0) return WERSA_OK;
  if (!x || !y || !scales || (residual && !r)) return WERSA_ERR_INVALID_ARG;
  const NormJob a{x, residual, weight, r, y, nullptr, scales, desc->rows, desc->stride_x, desc->stride_residual, desc->cols, desc->eps};
  return forward(*desc, a, true, (hipStream_t)hip_stream);
}

size_t wersa_rms_norm_workspace_bytes(const wersa_norm_desc *desc) {
  return validate(desc) == WERSA_OK ? (size_t)kBackGroups * desc->cols * sizeof(float) : 0;
}

wersa_status wersa_rms_norm_backward(const wersa_norm_desc *desc, const void *r, const float *weight, const float *rstd, const void *dy,
                                     const void *dr, void *dx, float *dweight, void *workspace, size_t workspace_bytes, void *hip_stream) {
  const wersa_status vs = validate(desc);
  if (vs != WERSA_OK) return vs;
  if (desc->rows > 0 && (!r || !rstd || !dy || !dx)) return WERSA_ERR_INVALID_ARG;
  if (dweight && (!workspace || workspace_bytes < wersa_rms_norm_workspace_bytes(desc) || misaligned(workspace, 256))) return WERSA_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)hip_stream;
  const NormBackJob a{r, dy, dr, weight, rstd, dx, dweight ? (float *)workspace : nullptr, desc->rows, desc->stride_x, desc->cols};
  int groups = 0;
  by_width(desc->cols, desc->dtype, [&](auto *type, auto lanes, auto pieces) {
    typedef typename std::remove_pointer<decltype(type)>::type T;
    constexpr int L = decltype(lanes)::value, P = decltype(pieces)::value;
    groups = (int)std::min<int64_t>(back_groups(P * 16 / sizeof(T)), (desc->rows + 256 / L - 1) / (256 / L));
    if (groups > 0) WERSA_STAGE("wersa_rms_norm_back", st, (norm_back_kernel<T, L, P><<<groups, 256, 0, st>>>(a)));
  });
  if (dweight)
    WERSA_STAGE("wersa_rms_norm_reduce", st, norm_reduce_kernel<<<(desc->cols + 15) / 16, 1024, 0, st>>>((const float *)workspace, groups, desc->cols, dweight));
  return hipGetLastError() == hipSuccess ? WERSA_OK : WERSA_ERR_LAUNCH;
}

}  // extern "C"
