// Entry points of the linear maps and of dropout: host checks, plan and dispatch.
// Contract: include/flashslice.h.
#include "fs_check.h"
#include "fs_internal.h"
#include "fs_linear.h"

#include <algorithm>
#include <cmath>

namespace fs {
namespace {

constexpr size_t kAlign = 256;
constexpr double kMaxValues = 1099511627776.0;  // 2^40

bool valid(const fs_linear* s) {
  if (!s || s->rows < 1 || s->Cin < 1 || s->Cout < 1) return false;
  if (s->dtype != FS_F32 && s->dtype != FS_BF16) return false;
  return (double)s->rows * (double)std::max(s->Cin, s->Cout) < kMaxValues;
}
bool supported(const fs_linear* s) { return s->Cin <= kLinearMaxC && s->Cout <= kLinearMaxC; }

bool valid_rows(const fs_rows* s) {
  if (!s || s->rows < 1 || s->C < 1) return false;
  if (s->dtype != FS_F32 && s->dtype != FS_BF16) return false;
  return (double)s->rows * (double)s->C < kMaxValues;
}

// The activation, and the dropout: p in [0, 1), with its generator if it drops anything.
bool valid_drop(int act, float p, const uint64_t* rng) {
  if (act < FS_ACT_NONE || act > FS_ACT_SILU) return false;
  return p >= 0.f && p < 1.f && (p == 0.f || rng);
}
uint32_t threshold_of(float p) { return (uint32_t)((double)p * 4294967296.0); }
float scale_of(float p) { return (float)(1.0 / (1.0 - (double)p)); }

size_t elem(int dtype) { return dtype == FS_BF16 ? 2 : 4; }
struct Sizes {
  size_t x, y, w, bias, dw;
};
Sizes sizes(const fs_linear* s) {
  const size_t e = elem(s->dtype), w = (size_t)s->Cout * s->Cin;
  return {(size_t)s->rows * s->Cin * e, (size_t)s->rows * s->Cout * e, w * e, (size_t)s->Cout * 4, w * 4};
}

LinearProblem problem(const fs_linear* s, int op, const void* a, const void* b, void* ws = nullptr, bool reset = true) {
  uint32_t* w = static_cast<uint32_t*>(ws);
  if (op == kLinFwd) return {op, s->dtype, s->rows, s->Cout, s->Cin, a, b, w, reset};
  if (op == kLinDx) return {op, s->dtype, s->rows, s->Cin, s->Cout, a, b, w, reset};
  return {op, s->dtype, s->Cout, s->Cin, s->rows, a, b, w, reset};
}
LinearPlan plan_of(const fs_linear* s, int op) {
  const LinearProblem p = problem(s, op, nullptr, nullptr);
  return linear_plan(op, p.dtype, p.M, p.N, p.K, true);
}
cudaError_t run(const LinearProblem& p, const LinearPlan& plan, const LinearEnd& e, char* scratch, cudaStream_t st) {
  return linear_simt(p, plan, e, scratch, st);
}
// [p, n] or nothing where p is one of the buffers that a call may update in place.
Span unless(const void* p, size_t n, const void* same) { return {p == same ? nullptr : p, n}; }

}  // namespace

LinearPlan linear_plan(int op, int dtype, int64_t M, int N, int64_t K, bool aligned) {
  LinearPlan p{};
  const int64_t tiles = ((M + 63) / 64) * ((N + 63) / 64);
  // Sums are split until the blocks fill the device twice, into parts of at least 64 terms.
  int64_t splits = std::max<int64_t>(1, std::min<int64_t>(2LL * num_sms() / tiles, (K + 63) / 64));
  p.per = ((K + splits - 1) / splits + 15) / 16 * 16;
  p.splits = (int)((K + p.per - 1) / p.per);
  if (p.splits > 1)
    p.part = ((size_t)p.splits * M * (((size_t)N + 3) & ~(size_t)3) + (op == kLinDw ? (size_t)p.splits * M : 0)) * 4;
  p.total = align_up(p.part, kAlign);
  return p;
}

}  // namespace fs

using namespace fs;

#define FS_CHECK_LINEAR(s)                        \
  do {                                            \
    if (!valid(s)) return FS_ERR_INVALID;         \
    if (!supported(s)) return FS_ERR_UNSUPPORTED; \
  } while (0)
#define FS_CHECK_ROWS(s)                                        \
  do {                                                          \
    if (!valid_rows(s)) return FS_ERR_INVALID;                  \
    if ((s)->C > kLinearMaxC) return FS_ERR_UNSUPPORTED;        \
  } while (0)

extern "C" {

size_t fs_linear_workspace_bytes(const fs_linear* s, int backward) {
  if (!valid(s) || !supported(s)) return 0;
  if (!backward) return kAlign + plan_of(s, kLinFwd).total;
  return kAlign + plan_of(s, kLinDx).total + plan_of(s, kLinDw).total;
}

int fs_linear_path_for_shape(const fs_linear* s, int backward) {
  if (!valid(s) || !supported(s)) return -1;
  return backward ? plan_of(s, kLinDx).path : plan_of(s, kLinFwd).path;
}

fs_status fs_linear_fwd(const fs_linear* s, const void* x, const void* W, const float* bias, int act, float p,
                        const uint64_t* rng, const void* res, void* y, void* pre, void* ws, size_t ws_bytes,
                        fs_stream_t stream) {
  FS_CHECK_LINEAR(s);
  if (!valid_drop(act, p, rng)) return FS_ERR_INVALID;
  FS_CHECK_PTR(x); FS_CHECK_PTR(W); FS_CHECK_PTR(y); FS_CHECK_PTR(ws);
  FS_CHECK_OPT(bias); FS_CHECK_OPT(rng); FS_CHECK_OPT(res); FS_CHECK_OPT(pre);
  const LinearPlan plan = plan_of(s, kLinFwd);
  const size_t need = kAlign + plan.total;
  if (ws_bytes < need) return FS_ERR_INVALID;
  const Sizes z = sizes(s);
  if (!disjoint({{x, z.x}, {W, z.w}, {bias, z.bias}, {rng, 16}, unless(res, z.y, y)}, {{y, z.y}, {pre, z.y}, {ws, need}}) ||
      !disjoint({{res, z.y}}, {{pre, z.y}, {ws, need}}))
    return FS_ERR_INVALID;
  LinearEnd e{};
  e.bias = bias; e.act = act; e.rng = p > 0.f ? rng : nullptr; e.threshold = threshold_of(p); e.scale = scale_of(p);
  e.res = res; e.y = y; e.pre_out = pre;
  return cuda_status(run(problem(s, kLinFwd, x, W, ws), plan, e, static_cast<char*>(ws) + kAlign,
                         reinterpret_cast<cudaStream_t>(stream)));
}

fs_status fs_linear_bwd(const fs_linear* s, const void* x, const void* W, const void* g, int act, float p,
                        const uint64_t* rng, const void* pre, const void* dres, void* dx, float* dW, float* dbias,
                        int accumulate, void* ws, size_t ws_bytes, fs_stream_t stream) {
  FS_CHECK_LINEAR(s);
  if (!valid_drop(act, p, rng)) return FS_ERR_INVALID;
  FS_CHECK_PTR(g); FS_CHECK_PTR(ws);
  FS_CHECK_OPT(x); FS_CHECK_OPT(W); FS_CHECK_OPT(rng); FS_CHECK_OPT(pre); FS_CHECK_OPT(dres); FS_CHECK_OPT(dx);
  FS_CHECK_OPT(dW); FS_CHECK_OPT(dbias);
  // dx needs W, and pre behind an activation; dW needs x; dbias comes with dW; one of the two is wanted
  if ((!dx && !dW) || (dx && !W) || (dx && act != FS_ACT_NONE && !pre) || (dW && !x) || (dbias && !dW) || (dres && !dx))
    return FS_ERR_INVALID;
  const LinearPlan plan_x = plan_of(s, kLinDx), plan_w = plan_of(s, kLinDw);
  const size_t need = kAlign + plan_x.total + plan_w.total;
  if (ws_bytes < need) return FS_ERR_INVALID;
  const Sizes z = sizes(s);
  if (!disjoint({{x, z.x}, {W, z.w}, {g, z.y}, {rng, 16}, {pre, z.x}, unless(dres, z.x, dx)},
                {{dx, z.x}, {dW, z.dw}, {dbias, z.bias}, {ws, need}}) ||
      !disjoint({{dres, z.x}}, {{dW, z.dw}, {dbias, z.bias}, {ws, need}}))
    return FS_ERR_INVALID;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  char* scratch = static_cast<char*>(ws) + kAlign;
  if (dx) {
    LinearEnd e{};
    e.act = act; e.rng = p > 0.f ? rng : nullptr; e.threshold = threshold_of(p); e.scale = scale_of(p);
    e.pre_in = pre; e.res = dres; e.y = dx;
    FS_CUDA(run(problem(s, kLinDx, g, W, ws), plan_x, e, scratch, st));
  }
  if (dW) {
    LinearEnd e{};
    e.y = dW; e.sums = dbias; e.accumulate = accumulate;
    FS_CUDA(run(problem(s, kLinDw, g, x, ws, !dx), plan_w, e, scratch + plan_x.total, st));
  }
  return FS_OK;
}

fs_status fs_dropout_fwd(const fs_rows* s, const void* x, int act, float p, const uint64_t* rng, const void* res, void* y,
                         fs_stream_t stream) {
  FS_CHECK_ROWS(s);
  if (!valid_drop(act, p, rng)) return FS_ERR_INVALID;
  FS_CHECK_PTR(x); FS_CHECK_PTR(y); FS_CHECK_OPT(rng); FS_CHECK_OPT(res);
  const size_t n = (size_t)s->rows * s->C * elem(s->dtype);
  if (!disjoint({unless(x, n, y), unless(res, n, y), {rng, 16}}, {{y, n}})) return FS_ERR_INVALID;
  DropArgs a{};
  a.x = x; a.res = res; a.y = y; a.rng = p > 0.f ? rng : nullptr; a.threshold = threshold_of(p); a.scale = scale_of(p);
  a.act = act; a.dtype = s->dtype; a.rows = s->rows; a.C = s->C;
  return cuda_status(dropout(a, reinterpret_cast<cudaStream_t>(stream)));
}

fs_status fs_dropout_bwd(const fs_rows* s, const void* dy, int act, float p, const uint64_t* rng, const void* pre,
                         void* dx, fs_stream_t stream) {
  FS_CHECK_ROWS(s);
  if (!valid_drop(act, p, rng)) return FS_ERR_INVALID;
  if (act != FS_ACT_NONE && !pre) return FS_ERR_INVALID;
  FS_CHECK_PTR(dy); FS_CHECK_PTR(dx); FS_CHECK_OPT(rng); FS_CHECK_OPT(pre);
  const size_t n = (size_t)s->rows * s->C * elem(s->dtype);
  if (!disjoint({unless(dy, n, dx), unless(pre, n, dx), {rng, 16}}, {{dx, n}})) return FS_ERR_INVALID;
  DropArgs a{};
  a.x = dy; a.pre = pre; a.y = dx; a.rng = p > 0.f ? rng : nullptr; a.threshold = threshold_of(p); a.scale = scale_of(p);
  a.act = act; a.dtype = s->dtype; a.backward = 1; a.rows = s->rows; a.C = s->C;
  return cuda_status(dropout(a, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
