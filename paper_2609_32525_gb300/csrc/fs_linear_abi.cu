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
  return linear_plan(op, p.dtype, p.M, p.N, p.K);
}
cudaError_t run(LinearProblem p, const LinearPlan& plan, const LinearEnd& e, char* scratch, cudaStream_t st) {
  return plan.path ? linear_tc(p, plan, e, scratch, st) : linear_simt(p, plan, e, scratch, st);
}

// A call's scratch: the status word, the operands that tensor cores cannot take as they are, and the parts
// of split sums.
struct Scratch {
  size_t need = kAlign;
  LinearPack packs[3];
  int n = 0;
  int dtype;
  explicit Scratch(int dtype_) : dtype(dtype_) {}
  // Where a product finds operand p: itself, or (from at()) its packed form.
  void pack(bool tc, const void* p, int64_t rows, int C) {
    if (!tc || !linear_packed(dtype, C)) return;
    packs[n++] = {p, reinterpret_cast<void*>(need), rows, C};
    need += align_up(linear_pack_bytes(rows, C), kAlign);
  }
  size_t add(size_t bytes) {
    need += bytes;
    return need - bytes;
  }
  cudaError_t launch(void* ws, cudaStream_t st) {
    for (int i = 0; i < n; i++) packs[i].dst = static_cast<char*>(ws) + reinterpret_cast<size_t>(packs[i].dst);
    return n ? linear_pack(packs, n, static_cast<uint32_t*>(ws), st) : cudaSuccess;
  }
  const void* at(bool tc, const void* p, int64_t rows, int C) const {
    for (int i = 0; tc && i < n; i++)
      if (packs[i].src == p && packs[i].rows == rows && packs[i].C == C) return packs[i].dst;
    return p;
  }
};
struct Plans {
  LinearPlan fwd, dx, dw;
  Scratch scratch;
  size_t at_fwd = 0, at_dx = 0, at_dw = 0;
};
// (The pointers of a size query are stand-ins.)
Plans plan_fwd(const fs_linear* s, const void* x, const void* W) {
  Plans p{plan_of(s, kLinFwd), {}, {}, Scratch(s->dtype)};
  p.scratch.pack(p.fwd.path, x, s->rows, s->Cin);
  p.scratch.pack(p.fwd.path, W, s->Cout, s->Cin);
  p.at_fwd = p.scratch.add(p.fwd.total);
  return p;
}
// dx, dw: wanted.  What a call does not want it does not pack, but its workspace has room for it.
Plans plan_bwd(const fs_linear* s, bool dx, bool dw, const void* x, const void* W, const void* g) {
  Plans p{{}, plan_of(s, kLinDx), plan_of(s, kLinDw), Scratch(s->dtype)};
  const bool tx = dx && p.dx.path, tw = dw && p.dw.path;
  p.scratch.pack(tx || tw, g, s->rows, s->Cout);
  p.scratch.pack(tx, W, s->Cout, s->Cin);
  p.scratch.pack(tw, x, s->rows, s->Cin);
  p.at_dx = p.scratch.add(p.dx.total);
  p.at_dw = p.scratch.add(p.dw.total);
  return p;
}
// [p, n] or nothing where p is one of the buffers that a call may update in place.
Span unless(const void* p, size_t n, const void* same) { return {p == same ? nullptr : p, n}; }

}  // namespace

LinearPlan linear_plan(int op, int dtype, int64_t M, int N, int64_t K) {
  LinearPlan p{};
  const double work = (double)M * N * (double)K;
  // Below this many products of terms a block's start and the two CTAs' hand-overs cost more than multiply-adds (1024
  // rows of 64 -> 64 bf16: 17 us against 13, of 256 -> 256 fp32: 23 against 17, backward 49 against 25).
  // Few channels fill a tile badly, but bf16 calls of them are bound by HBM (1,048,576 x 256 -> 4: forward 1093 us in
  // multiply-adds and 123 here, dx 481 and 145, dW 1968 and 130).
  const double least = dtype == FS_BF16 ? 16777216.0 : 134217728.0;
  // fp32 rows are split into parts by 64 terms and multiplied by 128 columns, however few there are.  What one tile of
  // multiply-adds holds, 64 columns and short sums (dW: 64 columns and 64 rows), takes less in those (1,048,576 rows, us
  // there, here: forward 2 -> 64 135, 244, 32 -> 64 183, 249, 64 -> 64 291, 249; dx of 64 from 3 119, 197, from 64 293, 181; dW of 64 x 64
  // 306, 473, of 128 x 64 598, 477), and a first map of few channels as much or less: 3 -> 256 527, 528, with GELU 725, 848; 2 -> 128 266,
  // 246 and 365, 424.
  const bool narrow = dtype == FS_F32 && (op == kLinDw ? M <= 64 && N <= 64 : (N <= 64 && K <= 32) || (op == kLinFwd && K < 16));
  const bool large = work >= least && !narrow && std::max(M, K) < (1LL << 31) - 512;
  // Few rows of a forward have a kernel that reads W once for four of them, 16 columns a block.  Where that is a block an SM or
  // more it is taken up to kLinearFew rows; with fewer, its time is the rows times the terms, and past a limit the
  // other path is faster (us here, there): bf16 2048 -> 2048, 4 rows 9.1, 11.4, 5 rows 12.2, 11.4; 4096 -> 1024, 2 rows
  // 9.6, 11.5, 3 rows 12.7, 11.6, 8 rows 29, 11.7; where the other path are multiply-adds: fp32 4096 -> 1024, 4 rows 20, 27, 6 rows
  // 33, 27; bf16 8192 -> 256, 2 rows 17, 18, 7 rows 50, 18.
  p.few = op == kLinFwd && M <= kLinearFew && (M * K <= (large ? 8192 : 16384) || N >= 16 * num_sms());
  // (dx of 4 rows of 1024, 4096 channels of g: 29 us in multiply-adds and 11 here, of 8 rows of 8192, 8192: 530 and 36;
  // fp32 437 and 238.)
  p.path = large && !p.few;
  int64_t splits;
  if (p.path) {
    // Pairs of CTAs take tiles; where there are fewer than half as many tiles, sums are split into parts of
    // at least 512 terms.
    const int bn = linear_tile_n(N, op != kLinFwd, dtype == FS_F32);
    const int64_t tiles = ((M + 255) / 256) * ((N + bn - 1) / bn), pairs = num_sms() / 2;
    splits = std::max<int64_t>(1, std::min<int64_t>(pairs / tiles, K / 512));
    p.per = ((K + splits - 1) / splits + 63) / 64 * 64;
  } else {
    // Sums are split until the blocks fill the device twice, into parts of at least 128 terms: below, a launch for the
    // join takes longer than the terms (backward of 100 x 64 x 66: 14.4 us with a split of its 100 rows and two
    // launches more, 10.1 without).
    const int64_t tiles = ((M + 63) / 64) * ((N + 63) / 64);
    splits = std::max<int64_t>(1, std::min<int64_t>(2LL * num_sms() / tiles, (K + 127) / 128));
    if (p.few) splits = 1;
    p.per = ((K + splits - 1) / splits + 15) / 16 * 16;
  }
  p.splits = (int)((K + p.per - 1) / p.per);
  if (p.splits > 1)
    p.part = ((size_t)p.splits * M * (((size_t)N + 3) & ~(size_t)3) + (op == kLinDw ? (size_t)p.splits * M : 0)) * 4;
  // dW: the parts of dbias behind them
  p.total = align_up(p.part, kAlign) + (op == kLinDw && p.path ? align_up((size_t)M * kLinearSumParts * 4, kAlign) : 0);
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
  return backward ? plan_bwd(s, true, true, nullptr, nullptr, nullptr).scratch.need
                  : plan_fwd(s, nullptr, nullptr).scratch.need;
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
  Plans plan = plan_fwd(s, x, W);
  const size_t need = plan.scratch.need;
  if (ws_bytes < need) return FS_ERR_INVALID;
  const Sizes z = sizes(s);
  if (!disjoint({{x, z.x}, {W, z.w}, {bias, z.bias}, {rng, 16}, unless(res, z.y, y)}, {{y, z.y}, {pre, z.y}, {ws, need}}) ||
      !disjoint({{res, z.y}}, {{pre, z.y}, {ws, need}}))
    return FS_ERR_INVALID;
  LinearEnd e{};
  e.bias = bias; e.act = act; e.rng = p > 0.f ? rng : nullptr; e.threshold = threshold_of(p); e.scale = scale_of(p);
  e.res = res; e.y = y; e.pre_out = pre;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const bool tc = plan.fwd.path;
  FS_CUDA(plan.scratch.launch(ws, st));
  return cuda_status(run(problem(s, kLinFwd, plan.scratch.at(tc, x, s->rows, s->Cin), plan.scratch.at(tc, W, s->Cout, s->Cin), ws, plan.scratch.n == 0),
                         plan.fwd, e, static_cast<char*>(ws) + plan.at_fwd, st));
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
  const size_t need = fs_linear_workspace_bytes(s, 1);
  if (ws_bytes < need) return FS_ERR_INVALID;
  const Sizes z = sizes(s);
  if (!disjoint({{x, z.x}, {W, z.w}, {g, z.y}, {rng, 16}, {pre, z.x}, unless(dres, z.x, dx)},
                {{dx, z.x}, {dW, z.dw}, {dbias, z.bias}, {ws, need}}) ||
      !disjoint({{dres, z.x}}, {{dW, z.dw}, {dbias, z.bias}, {ws, need}}))
    return FS_ERR_INVALID;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  Plans plan = plan_bwd(s, dx != nullptr, dW != nullptr, x, W, g);
  char* w = static_cast<char*>(ws);
  FS_CUDA(plan.scratch.launch(ws, st));
  LinearEnd ex{}, ew{};
  ex.act = act; ex.rng = p > 0.f ? rng : nullptr; ex.threshold = threshold_of(p); ex.scale = scale_of(p);
  ex.pre_in = pre; ex.res = dres; ex.y = dx;
  ew.y = dW; ew.sums = dbias; ew.accumulate = accumulate;
  const bool tx = plan.dx.path, tw = plan.dw.path, reset = plan.scratch.n == 0;
  const LinearProblem px = problem(s, kLinDx, plan.scratch.at(tx, g, s->rows, s->Cout), plan.scratch.at(tx, W, s->Cout, s->Cin), ws, reset);
  const LinearProblem pw = problem(s, kLinDw, plan.scratch.at(tw, g, s->rows, s->Cout), plan.scratch.at(tw, x, s->rows, s->Cin), ws,
                                   reset && !dx);
  // (a grid of both products' tiles has to stay below 2^31 blocks)
  if (dx && dW && !tx && !tw && s->rows < (1LL << 30))
    return cuda_status(linear_simt_bwd(px, plan.dx, ex, w + plan.at_dx, pw, plan.dw, ew, w + plan.at_dw, st));
  if (dx) FS_CUDA(run(px, plan.dx, ex, w + plan.at_dx, st));
  if (dW) FS_CUDA(run(pw, plan.dw, ew, w + plan.at_dw, st));
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
