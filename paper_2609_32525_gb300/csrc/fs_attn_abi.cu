// Entry points of the token attention: host checks, workspace layout, dispatch.  Contract:
// include/flashslice.h.
#include "fs_attn.h"
#include "fs_attn_tc.h"
#include "fs_check.h"
#include "fs_internal.h"

#include <cfloat>
#include <cmath>

namespace fs {
namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMostTokens = 1 << 20;

// The cap as the kernels apply it, cap tanh(q.k scale / cap): not at all where scale / cap is below
// fp32's normal range, whose few bits would round every score.  There tanh(x) is x (to 2^-25 of it
// for products up to 2^114), and c is s.
float applied_cap(const fs_attn_shape* s) {
  return s->cap > 0.f && std::fabs(s->scale / s->cap) < FLT_MIN ? 0.f : s->cap;
}
bool valid(const fs_attn_shape* s) {
  if (!s || s->B < 1 || s->H < 1 || s->Hkv < 1 || s->Gq < 1 || s->Gk < 1 || s->d < 1) return false;
  if (s->H % s->Hkv != 0) return false;
  if (s->mask != FS_MASK_NONE && s->mask != FS_MASK_PREFIX) return false;
  if (s->mask == FS_MASK_PREFIX && s->Gq > s->Gk) return false;
  if (!std::isfinite(s->scale) || !(s->cap >= 0.f) || !std::isfinite(s->cap)) return false;
  // the kernels' factors
  const float cap = applied_cap(s);
  if (!std::isfinite(cap > 0.f ? s->scale / cap : s->scale * kLog2e) || !std::isfinite(cap * kLog2e)) return false;
  const double most = (double)s->B * s->H * (double)(s->Gq > s->Gk ? s->Gq : s->Gk) * s->d;
  return most < 1099511627776.0;  // 2^40
}
bool supported(const fs_attn_shape* s) {
  return (s->d == 16 || s->d == 32 || s->d == 64) && s->B * s->H <= 65535 && s->Gk <= kMostTokens &&
         (int64_t)(s->H / s->Hkv) * s->Gq <= kMostTokens;
}

struct Dims {
  int64_t units, rows, nq, nk;  // nq, nk: floats of q and of k
};
Dims dims(const fs_attn_shape* s) {
  Dims n;
  n.units = s->B * s->Hkv;
  n.rows = (int64_t)(s->H / s->Hkv) * s->Gq;
  n.nq = n.units * n.rows * s->d;
  n.nk = n.units * s->Gk * s->d;
  return n;
}

struct Layout {
  AttnPlan plan;
  size_t delta, part, part_kv, total;
  // of the tensor-core kernels: images by tensor (k, v, q, dout), of rows and of columns
  size_t row_img[4], col_img[4], k_pos, k_doc, k_range, q_info, q_tok, q_range;
  int64_t rows_pad, k_pad;
};
Layout layout(const fs_attn_shape* s, bool backward) {
  const Dims n = dims(s);
  Layout l{};
  l.plan = attn_plan(n.units, n.rows, s->Gk, s->d, backward);
  const AttnPlan& p = l.plan;
  size_t off = kAlign;  // the status word
  auto take = [&](int64_t floats) {
    const size_t o = off;
    off = align_up(off + (size_t)floats * 4, kAlign);
    return o;
  };
  if (backward) {
    l.delta = take(p.delta ? n.units * n.rows : 0);
    l.part = take(p.splits > 1 ? p.splits * n.nq : 0);
    l.part_kv = take(p.splits_kv > 1 ? p.splits_kv * 2 * n.nk : 0);
  } else {
    l.part = take(p.splits > 1 ? p.splits * (n.nq + 2 * n.units * n.rows) : 0);
  }
  if (p.tc) {
    l.k_pad = (s->Gk + 63) / 64 * 64;
    l.rows_pad = (n.rows + 63) / 64 * 64;
    // forward: rows of k, columns of v; backward: rows of all four, columns of k, q and dout
    for (int t = 0; t < (backward ? 4 : 2); t++) {
      const int64_t img = 2 * n.units * (t < 2 ? l.k_pad : l.rows_pad) * (s->d < 32 ? 32 : s->d);
      l.row_img[t] = backward || t == 0 ? take(img) : 0;
      l.col_img[t] = backward == (t != 1) ? take(img) : 0;
    }
    l.k_pos = take(s->B * l.k_pad);
    l.k_doc = take(s->B * l.k_pad);
    l.k_range = take(2 * s->B * (l.k_pad / 32));
    if (backward) {
      l.q_info = take(4 * n.units * l.rows_pad);
      l.q_tok = take(2 * n.units * l.rows_pad);
      l.q_range = take(2 * n.units * (l.rows_pad / 32));
    }
  }
  l.total = off;
  return l;
}

float* at(void* ws, size_t off) { return reinterpret_cast<float*>(static_cast<char*>(ws) + off); }

// What a mask may hold: positions only with slopes, both sides' or neither's; documents of
// both sides or neither; prefixes only under the prefix mask.
fs_status check_mask(const fs_attn_shape* s, const fs_attn_mask* m) {
  const void* all[] = {m->slopes, m->pos_q, m->pos_k, m->doc_q, m->doc_k, m->prefix};
  for (const void* p : all)  // read word by word: a view of a longer array will do
    if (reinterpret_cast<uintptr_t>(p) & 3u) return FS_ERR_INVALID;
  if (!m->pos_q != !m->pos_k || !m->doc_q != !m->doc_k) return FS_ERR_INVALID;
  if ((m->pos_q && !m->slopes) || (m->prefix && s->mask != FS_MASK_PREFIX)) return FS_ERR_INVALID;
  return FS_OK;
}

// No output may share a byte with anything that the call reads or with another output.
bool apart(const fs_attn_shape* s, const fs_attn_mask& m, std::initializer_list<Span> ins,
           std::initializer_list<Span> outs) {
  const size_t bq = (size_t)s->B * s->Gq * 4, bk = (size_t)s->B * s->Gk * 4;
  return disjoint(ins, outs) && disjoint({{m.slopes, (size_t)s->H * 4}, {m.pos_q, bq}, {m.pos_k, bk}, {m.doc_q, bq},
                                          {m.doc_k, bk}, {m.prefix, (size_t)s->B * 4}},
                                         outs);
}

AttnArgs args_of(const fs_attn_shape* s, const fs_attn_mask& m, const float* q, const float* k, const float* v,
                 void* ws, const Layout& l, bool backward) {
  const Dims n = dims(s);
  const AttnPlan& p = l.plan;
  AttnArgs a{};
  a.q = q; a.k = k; a.v = v;
  a.slopes = m.slopes; a.pos_q = m.pos_q; a.pos_k = m.pos_k;
  a.doc_q = m.doc_q; a.doc_k = m.doc_k; a.prefix = m.prefix;
  a.B = (int)s->B; a.H = s->H; a.Hkv = s->Hkv; a.Gq = s->Gq; a.Gk = s->Gk;
  a.rows = (int)n.rows; a.units = (int)n.units;
  a.causal = s->mask == FS_MASK_PREFIX;
  a.warps = p.warps; a.splits = p.splits; a.splits_kv = p.splits_kv;
  a.scale = s->scale; a.cap = applied_cap(s);
  a.status = static_cast<uint32_t*>(ws);
  a.part = at(ws, l.part);
  if (backward) {
    a.delta = p.delta ? at(ws, l.delta) : nullptr;
    a.part_kv = at(ws, l.part_kv);
  }
  return a;
}

cudaError_t run(const fs_attn_shape* s, const AttnArgs& a, void* ws, const Layout& l, bool backward, cudaStream_t st) {
  if (!l.plan.tc) return backward ? attn_bwd(a, s->d, st) : attn_fwd(a, s->d, st);
  AttnTcArgs t{};
  t.a = a;
  for (int i = 0; i < 4; i++) {
    t.row_img[i] = l.row_img[i] ? reinterpret_cast<uint8_t*>(at(ws, l.row_img[i])) : nullptr;
    t.col_img[i] = l.col_img[i] ? reinterpret_cast<uint8_t*>(at(ws, l.col_img[i])) : nullptr;
  }
  t.k_pos = at(ws, l.k_pos);
  t.k_doc = reinterpret_cast<int*>(at(ws, l.k_doc));
  t.k_range = reinterpret_cast<int2*>(at(ws, l.k_range));
  t.q_info = at(ws, l.q_info);
  t.q_tok = reinterpret_cast<int*>(at(ws, l.q_tok));
  t.q_range = reinterpret_cast<int2*>(at(ws, l.q_range));
  t.rows_pad = (int)l.rows_pad;
  t.k_pad = (int)l.k_pad;
  return s->d == 16 ? attn_tc<16>(t, backward, st) : s->d == 32 ? attn_tc<32>(t, backward, st) : attn_tc<64>(t, backward, st);
}

}  // namespace
}  // namespace fs

using namespace fs;

#define FS_CHECK_ATTN(s)                          \
  do {                                            \
    if (!valid(s)) return FS_ERR_INVALID;         \
    if (!supported(s)) return FS_ERR_UNSUPPORTED; \
  } while (0)

extern "C" {

size_t fs_attn_workspace_bytes(const fs_attn_shape* s, int backward) {
  if (!valid(s) || !supported(s)) return 0;
  return layout(s, backward != 0).total;
}

int fs_attn_path_for_shape(const fs_attn_shape* s, int backward) {
  if (!valid(s) || !supported(s)) return -1;
  return layout(s, backward != 0).plan.tc ? 1 : 0;
}

fs_status fs_attn_fwd(const fs_attn_shape* s, const float* q, const float* k, const float* v,
                      const fs_attn_mask* mask, float* out, float* lse, void* ws, size_t ws_bytes,
                      fs_stream_t stream) {
  FS_CHECK_ATTN(s);
  FS_CHECK_PTR(q); FS_CHECK_PTR(k); FS_CHECK_PTR(v); FS_CHECK_PTR(out); FS_CHECK_PTR(lse); FS_CHECK_PTR(ws);
  const fs_attn_mask m = mask ? *mask : fs_attn_mask{};
  if (fs_status e = check_mask(s, &m)) return e;
  const Dims n = dims(s);
  const Layout l = layout(s, false);
  const size_t rb = (size_t)n.units * n.rows * 4, qb = (size_t)n.nq * 4, kb = (size_t)n.nk * 4;
  if (ws_bytes < l.total) return FS_ERR_INVALID;
  if (!apart(s, m, {{q, qb}, {k, kb}, {v, kb}}, {{out, qb}, {lse, rb}, {ws, l.total}})) return FS_ERR_INVALID;
  AttnArgs a = args_of(s, m, q, k, v, ws, l, false);
  a.out = out; a.lse = lse;
  return cuda_status(run(s, a, ws, l, false, reinterpret_cast<cudaStream_t>(stream)));
}

fs_status fs_attn_bwd(const fs_attn_shape* s, const float* q, const float* k, const float* v,
                      const fs_attn_mask* mask, const float* out, const float* lse, const float* dout, float* dq,
                      float* dk, float* dv, void* ws, size_t ws_bytes, fs_stream_t stream) {
  FS_CHECK_ATTN(s);
  FS_CHECK_PTR(q); FS_CHECK_PTR(k); FS_CHECK_PTR(v); FS_CHECK_PTR(out); FS_CHECK_PTR(lse); FS_CHECK_PTR(dout);
  FS_CHECK_PTR(dq); FS_CHECK_PTR(dk); FS_CHECK_PTR(dv); FS_CHECK_PTR(ws);
  const fs_attn_mask m = mask ? *mask : fs_attn_mask{};
  if (fs_status e = check_mask(s, &m)) return e;
  const Dims n = dims(s);
  const Layout l = layout(s, true);
  const size_t rb = (size_t)n.units * n.rows * 4, qb = (size_t)n.nq * 4, kb = (size_t)n.nk * 4;
  if (ws_bytes < l.total) return FS_ERR_INVALID;
  if (!apart(s, m, {{q, qb}, {k, kb}, {v, kb}, {out, qb}, {lse, rb}, {dout, qb}},
             {{dq, qb}, {dk, kb}, {dv, kb}, {ws, l.total}}))
    return FS_ERR_INVALID;
  AttnArgs a = args_of(s, m, q, k, v, ws, l, true);
  a.out = const_cast<float*>(out); a.lse = const_cast<float*>(lse); a.dout = dout;
  a.dq = dq; a.dk = dk; a.dv = dv;
  return cuda_status(run(s, a, ws, l, true, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
