// Rows rounded to int8 with a scale each: tokens on their way into an 8-bit product, the rows of a weight when it is laid out.
// q[t][c] = round(127 x[t][c] / a_t), s[t] = a_t / 127, a_t = max_c |x[t][c]| (rows_io.cuh says how the integer is the exact one).
//
// Bound by HBM: an element is read once and one byte is written.  A CTA takes a row and keeps it in registers between the maximum
// and the rounding, 8 CHUNKS elements a thread.
#include "rows_io.cuh"

namespace {

using namespace rows;

template <typename T, bool ALIGNED, int CHUNKS>
__global__ void __launch_bounds__(1024)
quantize_rows_kernel(const T* x, int64_t ldx, int64_t cols, int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale) {
  grid_begin();
  __shared__ float red[1][32];
  const int64_t row = blockIdx.x;
  const T* const xr = x + row * ldx;
  Raw8<T> raw[CHUNKS];
  unsigned top = 0;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * 8;
    raw[c] = e < cols ? row_load<ALIGNED>(xr, e, cols) : raw_zero<T>();
  }
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) top = max(top, raw_top(raw[c]));
  const RowScale r = row_scale<sizeof(T) == 2>(cta_max(top, red));
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int64_t e = ((int64_t)c * blockDim.x + threadIdx.x) * 8;
    if (e < cols) {
      float v[8];
      raw_get(raw[c], v);
      *reinterpret_cast<uint2*>(q + row * ldq + e) = row_round8<sizeof(T) == 2>(v, r);     // (a row of q has room for the eight: ldq is a multiple of 16)
    }
  }
  if (threadIdx.x == 0) scale[row] = r.s;
}

// Rows longer than a CTA's registers hold: read twice, the second time from L2.
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(1024)
quantize_long_rows_kernel(const T* x, int64_t ldx, int64_t cols, int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale) {
  grid_begin();
  __shared__ float red[1][32];
  const int64_t row = blockIdx.x;
  const T* const xr = x + row * ldx;
  unsigned top = 0;
  for (int64_t e = threadIdx.x * 8; e < cols; e += 8 * blockDim.x) top = max(top, raw_top(row_load<ALIGNED>(xr, e, cols)));
  const RowScale r = row_scale<sizeof(T) == 2>(cta_max(top, red));
  for (int64_t e = threadIdx.x * 8; e < cols; e += 8 * blockDim.x) {
    float v[8];
    raw_get(row_load<ALIGNED>(xr, e, cols), v);
    *reinterpret_cast<uint2*>(q + row * ldq + e) = row_round8<sizeof(T) == 2>(v, r);
  }
  if (threadIdx.x == 0) scale[row] = r.s;
}

template <typename T, bool ALIGNED>
void launch_typed(const T* x, int64_t ldx, int64_t n, int64_t cols, int8_t* q, int64_t ldq, float* scale, cudaStream_t s) {
  const dim3 grid((unsigned)n);
  const int64_t units = (cols + 7) / 8;
  auto threads = [&](int chunks) { return dim3((unsigned)(((units + chunks - 1) / chunks + 31) / 32 * 32)); };
  // few rows: as many threads as the row has chunks; many: more of a row in flight per thread and fewer warps to meet at the barrier
  if (units <= 128 || (n <= 148 && units <= 1024)) launch_dependent(quantize_rows_kernel<T, ALIGNED, 1>, grid, threads(1), 0, s, x, ldx, cols, q, ldq, scale);
  else if (units <= 512) launch_dependent(quantize_rows_kernel<T, ALIGNED, 2>, grid, threads(2), 0, s, x, ldx, cols, q, ldq, scale);
  else if (units <= 4096) launch_dependent(quantize_rows_kernel<T, ALIGNED, 4>, grid, threads(4), 0, s, x, ldx, cols, q, ldq, scale);
  else launch_dependent(quantize_long_rows_kernel<T, ALIGNED>, grid, dim3(1024), 0, s, x, ldx, cols, q, ldq, scale);
}

template <typename T>
void launch_by_alignment(const void* x, int64_t ldx, int64_t n, int64_t cols, int8_t* q, int64_t ldq, float* scale, cudaStream_t s) {
  const T* xt = static_cast<const T*>(x);
  if (aligned16(x, n > 1 ? ldx : 8, (int)sizeof(T))) launch_typed<T, true>(xt, ldx, n, cols, q, ldq, scale, s);
  else launch_typed<T, false>(xt, ldx, n, cols, q, ldq, scale, s);
}

}  // namespace

int rows_dtype_bytes(int32_t dtype) {
  return dtype == ARMOR_DTYPE_F32 ? 4 : (dtype == ARMOR_DTYPE_BF16 || dtype == ARMOR_DTYPE_F16 ? 2 : 0);
}

// q [n, ldq], scale [n] of x [n, cols]; up to 2^31 - 1 rows a launch
armor_status launch_quantize_rows(armor_ctx* c, const void* x, int32_t dtype, int64_t ldx, int64_t n, int64_t cols, int8_t* q,
                                  int64_t ldq, float* scale, cudaStream_t s) {
  const int64_t esize = rows_dtype_bytes(dtype);
  KTimer kt(c, ARMOR_KC_FORWARD, (double)n * (double)cols * (double)(esize + 1), s);
  for (int64_t r0 = 0; r0 < n; r0 += 0x7fffffff) {
    const int64_t m = n - r0 < 0x7fffffff ? n - r0 : 0x7fffffff;
    const void* xr = static_cast<const char*>(x) + r0 * ldx * esize;
    if (dtype == ARMOR_DTYPE_F32) launch_by_alignment<float>(xr, ldx, m, cols, q + r0 * ldq, ldq, scale + r0, s);
    else if (dtype == ARMOR_DTYPE_BF16) launch_by_alignment<__nv_bfloat16>(xr, ldx, m, cols, q + r0 * ldq, ldq, scale + r0, s);
    else launch_by_alignment<__half>(xr, ldx, m, cols, q + r0 * ldq, ldq, scale + r0, s);
    c->launches++;
  }
  return cudaGetLastError() == cudaSuccess ? ARMOR_OK : ARMOR_ERR_CUDA;
}
