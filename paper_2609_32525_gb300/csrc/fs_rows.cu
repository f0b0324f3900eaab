// Entry points of the layer norm and the 8-bit checkpoint: host checks and dispatch, and the
// fixed-order sum of the parameter gradients' partials.  Contract: include/flashslice.h.
#include "fs_check.h"
#include "fs_internal.h"
#include "fs_launch.h"
#include "fs_rows.h"

#include <cmath>
#include <cuda_bf16.h>

namespace fs {
namespace {

// Column sums of part [blocks][2 C] in a fixed order: 32 threads share a column's rows (thread
// y takes rows y, y + 32, ...), their sums are added in order.  Eight columns a block: a call has
// few columns, and what counts is how many loads are on their way.
__global__ void __launch_bounds__(256) k_norm_reduce(const float* __restrict__ part, int64_t blocks, int C,
                                                      float* __restrict__ dgamma, float* __restrict__ dbeta,
                                                      int accumulate) {
  __shared__ float sm[32][9];
  grid_begin(part);
  const int64_t n = 2LL * C, c = (int64_t)blockIdx.x * 8 + threadIdx.x;
  float s = 0.f;
  if (c < n) {
#pragma unroll 8
    for (int64_t b = threadIdx.y; b < blocks; b += 32) s += part[b * n + c];
  }
  sm[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y != 0 || c >= n) return;
  s = 0.f;
#pragma unroll
  for (int y = 0; y < 32; y++) s += sm[y][threadIdx.x];
  float* out = c < C ? dgamma + c : dbeta + (c - C);
  *out = accumulate ? *out + s : s;
}

constexpr size_t kAlign = 256;

bool valid_rows(const fs_rows* s) {
  if (!s || s->rows < 1 || s->C < 1) return false;
  if (s->dtype != FS_F32 && s->dtype != FS_BF16) return false;
  return (double)s->rows * (double)s->C < 1099511627776.0;  // 2^40
}
bool supported_rows(const fs_rows* s) { return s->C <= kRowsMaxC; }

int64_t bwd_blocks(const fs_rows* s) {
  return s->dtype == FS_BF16 ? norm_bwd_blocks<__nv_bfloat16>(s->rows, s->C) : norm_bwd_blocks<float>(s->rows, s->C);
}

struct Sizes {
  size_t data, row, q8, e8, par;
};
Sizes sizes(const fs_rows* s) {
  const size_t n = (size_t)s->rows * s->C;
  return {n * (s->dtype == FS_BF16 ? 2 : 4), (size_t)s->rows * 4, n,
          (size_t)s->rows * ((s->C + kCkptBlock - 1) / kCkptBlock), (size_t)s->C * 4};
}

// [p, n] or nothing where p is one of the buffers that a call may update in place.
Span unless(const void* p, size_t n, const void* same) { return {p == same ? nullptr : p, n}; }

}  // namespace
}  // namespace fs

using namespace fs;

#define FS_CHECK_ROWS(s)                               \
  do {                                                 \
    if (!valid_rows(s)) return FS_ERR_INVALID;         \
    if (!supported_rows(s)) return FS_ERR_UNSUPPORTED; \
  } while (0)

extern "C" {

size_t fs_norm_workspace_bytes(const fs_rows* s) {
  if (!valid_rows(s) || !supported_rows(s)) return 0;
  return kAlign + align_up((size_t)bwd_blocks(s) * 2 * s->C * sizeof(float), kAlign);
}

fs_status fs_norm_fwd(const fs_rows* s, const void* x, const void* res, const float* gamma, const float* beta,
                      float eps, void* sum, void* y, float* mean, float* rstd, int8_t* q8, uint8_t* e8,
                      fs_stream_t stream) {
  FS_CHECK_ROWS(s);
  if (!(eps >= 0.f) || !std::isfinite(eps)) return FS_ERR_INVALID;
  FS_CHECK_PTR(x); FS_CHECK_PTR(y);
  FS_CHECK_OPT(res); FS_CHECK_OPT(gamma); FS_CHECK_OPT(beta); FS_CHECK_OPT(sum); FS_CHECK_OPT(mean);
  FS_CHECK_OPT(rstd); FS_CHECK_OPT(q8); FS_CHECK_OPT(e8);
  if ((sum && !res) || !q8 != !e8) return FS_ERR_INVALID;
  const Sizes z = sizes(s);
  if (!disjoint({{x, z.data}, {res, z.data}, {gamma, z.par}, {beta, z.par}},
                {{y, z.data}, {mean, z.row}, {rstd, z.row}, {q8, z.q8}, {e8, z.e8}}) ||
      !disjoint({unless(x, z.data, sum), unless(res, z.data, sum), {gamma, z.par}, {beta, z.par}, {y, z.data},
                 {mean, z.row}, {rstd, z.row}, {q8, z.q8}, {e8, z.e8}},
                {{sum, z.data}}))
    return FS_ERR_INVALID;
  RowsArgs a{};
  a.x = x; a.res = res; a.gamma = gamma; a.beta = beta; a.eps = eps;
  a.sum = sum; a.y = y; a.mean = mean; a.rstd = rstd; a.q8 = q8; a.e8 = e8;
  a.rows = s->rows; a.C = s->C;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return cuda_status(s->dtype == FS_BF16 ? norm_fwd<__nv_bfloat16>(a, st) : norm_fwd<float>(a, st));
}

fs_status fs_norm_bwd(const fs_rows* s, const void* v, const int8_t* q8, const uint8_t* e8, const float* gamma,
                      const float* mean, const float* rstd, const void* dy, const void* dres, void* dv,
                      float* dgamma, float* dbeta, int accumulate, void* ws, size_t ws_bytes, fs_stream_t stream) {
  FS_CHECK_ROWS(s);
  if (!v == !q8 || !q8 != !e8 || !dgamma != !dbeta) return FS_ERR_INVALID;
  FS_CHECK_OPT(v); FS_CHECK_OPT(q8); FS_CHECK_OPT(e8); FS_CHECK_OPT(gamma); FS_CHECK_OPT(dres);
  FS_CHECK_OPT(dgamma); FS_CHECK_OPT(dbeta);
  FS_CHECK_PTR(mean); FS_CHECK_PTR(rstd); FS_CHECK_PTR(dy); FS_CHECK_PTR(dv); FS_CHECK_PTR(ws);
  const size_t need = fs_norm_workspace_bytes(s);
  if (ws_bytes < need) return FS_ERR_INVALID;
  const Sizes z = sizes(s);
  if (!disjoint({{v, z.data}, {q8, z.q8}, {e8, z.e8}, {gamma, z.par}, {mean, z.row}, {rstd, z.row},
                 unless(dy, z.data, dv), unless(dres, z.data, dv)},
                {{dv, z.data}, {dgamma, z.par}, {dbeta, z.par}, {ws, need}}) ||
      !disjoint({{dy, z.data}, {dres, z.data}}, {{dgamma, z.par}, {dbeta, z.par}, {ws, need}}))
    return FS_ERR_INVALID;
  RowsArgs a{};
  a.x = v; a.q8 = const_cast<int8_t*>(q8); a.e8 = const_cast<uint8_t*>(e8);
  a.gamma = gamma; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.dy = dy; a.dres = dres; a.y = dv; a.dgamma = dgamma; a.dbeta = dbeta; a.accumulate = accumulate;
  a.rows = s->rows; a.C = s->C;
  a.status = static_cast<uint32_t*>(ws);
  a.part = dgamma ? reinterpret_cast<float*>(static_cast<char*>(ws) + kAlign) : nullptr;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  int64_t blocks = 0;
  FS_CUDA(s->dtype == FS_BF16 ? norm_bwd<__nv_bfloat16>(a, &blocks, st) : norm_bwd<float>(a, &blocks, st));
  if (dgamma)
    FS_CUDA(launch(k_norm_reduce, dim3((unsigned)((2LL * s->C + 7) / 8)), dim3(8, 32), 0, st, a.part, blocks, s->C,
                   dgamma, dbeta, accumulate));
  return FS_OK;
}

fs_status fs_ckpt_pack(const fs_rows* s, const void* x, int8_t* q8, uint8_t* e8, fs_stream_t stream) {
  FS_CHECK_ROWS(s);
  FS_CHECK_PTR(x); FS_CHECK_PTR(q8); FS_CHECK_PTR(e8);
  const Sizes z = sizes(s);
  if (!disjoint({{x, z.data}}, {{q8, z.q8}, {e8, z.e8}})) return FS_ERR_INVALID;
  RowsArgs a{};
  a.x = x; a.q8 = q8; a.e8 = e8; a.rows = s->rows; a.C = s->C;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return cuda_status(s->dtype == FS_BF16 ? ckpt_pack<__nv_bfloat16>(a, st) : ckpt_pack<float>(a, st));
}

fs_status fs_ckpt_unpack(const fs_rows* s, const int8_t* q8, const uint8_t* e8, void* x, fs_stream_t stream) {
  FS_CHECK_ROWS(s);
  FS_CHECK_PTR(x); FS_CHECK_PTR(q8); FS_CHECK_PTR(e8);
  const Sizes z = sizes(s);
  if (!disjoint({{q8, z.q8}, {e8, z.e8}}, {{x, z.data}})) return FS_ERR_INVALID;
  RowsArgs a{};
  a.q8 = const_cast<int8_t*>(q8); a.e8 = const_cast<uint8_t*>(e8); a.y = x; a.rows = s->rows; a.C = s->C;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  return cuda_status(s->dtype == FS_BF16 ? ckpt_unpack<__nv_bfloat16>(a, st) : ckpt_unpack<float>(a, st));
}

}  // extern "C"
