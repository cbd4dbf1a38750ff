// C ABI of the heads' norms with rotation: argument validation and dispatch to the HIP
// launchers.  Every argument check runs before the first HIP call of an entry point.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "tcu.h"
#include "tcu_heads.h"
#include "tcu_host.h"
#include "tcu_operand.h"

#define TCU_EXPORT extern "C" __attribute__((visibility("default")))

namespace {

using namespace tcu;

struct Sizes {
  int64_t tokens, hq, hk, dim, rot;
  float eps;
  int flags, elem;
};

int check_sizes(const Sizes &s) {
  if (!elem_ok(s.elem) || (s.flags & ~TCU_ROPE_ADJACENT) != 0) return TCU_ERR_UNSUPPORTED;
  if (!dim_ok(s.tokens) || s.hq < 0 || s.hk < 0 || s.hq > TCU_MAX_HEADS || s.hk > TCU_MAX_HEADS ||
      s.dim < 1 || s.dim > TCU_MAX_HEAD_DIM || s.rot < 0 || s.rot > s.dim || s.rot % 2 != 0 ||
      !(s.eps >= 0.f) || std::isinf(s.eps))
    return TCU_ERR_SHAPE;
  return TCU_OK;
}

// tokens x heads x dim elements as a view of rows: the outer of the two indices, and
// the extent of the inner one with its runs of `dim`.
Operand heads_view(const Heads &h, int64_t heads, const Sizes &s, bool out = false) {
  Operand o{h.p, 0, 0, 0, elem_size(s.elem), (int)elem_size(s.elem), out};
  if (s.tokens == 0 || heads == 0) return o;
  const bool by_token = heads == 1 || (s.tokens > 1 && h.hd <= h.ld);
  const int64_t outer = by_token ? h.ld : h.hd, inner = by_token ? h.hd : h.ld;
  const int64_t inner_n = by_token ? heads : s.tokens;
  o.rows = by_token ? s.tokens : heads;
  o.cols = s.dim;
  if (inner_n > 1) {
    // (an inner pitch in which the elements do not fit is given as one of too many columns)
    const __int128 extent = (__int128)(inner_n - 1) * inner + s.dim;
    o.cols = inner < s.dim || extent >= kMaxExtent ? kMaxExtent : (int64_t)extent;
    o.runs = inner_n;
    o.run = s.dim;
    o.step = inner;
  }
  o.ld = o.rows > 1 ? outer : o.cols;
  return o;
}

bool same(const Heads &a, const Heads &b) { return a.p == b.p && a.ld == b.ld && a.hd == b.hd; }

}  // namespace

TCU_EXPORT int tcu_qk_norm(const void *q, int64_t ldq, int64_t hdq, const void *k, int64_t ldk,
                           int64_t hdk, const void *wq, const void *wk, const float *freq,
                           const int32_t *pos, void *yq, int64_t ldyq, int64_t hdyq, void *yk,
                           int64_t ldyk, int64_t hdyk, int64_t tokens, int64_t hq, int64_t hk,
                           int64_t dim, int64_t rot, float eps, int flags, int elem,
                           void *hip_stream) {
  const Sizes s{tokens, hq, hk, dim, rot, eps, flags, elem};
  int rc = check_sizes(s);
  if (rc != TCU_OK) return rc;
  QkNormArgs a{};
  a.x[0] = Heads{q, ldq, hdq};
  a.x[1] = Heads{k, ldk, hdk};
  a.y[0] = Heads{yq, ldyq, hdyq};
  a.y[1] = Heads{yk, ldyk, hdyk};
  const bool any = tokens > 0 && hq + hk > 0;
  const int64_t es = elem_size(elem);
  const Operand ops[] = {heads_view(a.y[0], hq, s, true), heads_view(a.y[1], hk, s, true),
                         heads_view(a.x[0], hq, s), heads_view(a.x[1], hk, s),
                         vec(wq, any && hq > 0 ? dim : 0, es, 16),
                         vec(wk, any && hk > 0 ? dim : 0, es, 16),
                         vec(freq, any ? rot / 2 : 0, 4, 4), vec(pos, any && rot > 0 ? tokens : 0, 4, 4)};
  rc = check_operands(ops, {{same(a.y[0], a.x[0]) ? 0 : -1, 2}, {same(a.y[1], a.x[1]) ? 1 : -1, 3}});
  if (rc != TCU_OK) return rc;
  if (!any) return TCU_OK;
  int num_cus = 0;
  rc = device_ready(&num_cus);
  if (rc != TCU_OK) return rc;
  rc = check_device(ops);
  if (rc != TCU_OK) return rc;
  a.w[0] = wq;
  a.w[1] = wk;
  a.freq = freq;
  a.pos = pos;
  a.tokens = tokens;
  a.heads[0] = (int)hq;
  a.heads[1] = (int)hk;
  a.dim = (int)dim;
  a.rot = (int)rot;
  a.eps = eps;
  a.adjacent = (flags & TCU_ROPE_ADJACENT) != 0;
  return launch_qk_norm(elem, a, (hipStream_t)hip_stream, num_cus) == hipSuccess ? TCU_OK
                                                                                 : TCU_ERR_HIP;
}

TCU_EXPORT int64_t tcu_qk_norm_grad_work(int64_t tokens, int64_t hq, int64_t hk, int64_t dim) {
  const Sizes s{tokens, hq, hk, dim, 0, 0.f, 0, TCU_ELEM_F32};
  return check_sizes(s) == TCU_OK ? (int64_t)kHeadParts * 2 * dim * 4 : -1;
}

TCU_EXPORT int tcu_qk_norm_grad(const void *dyq, int64_t lddyq, int64_t hddyq, const void *dyk,
                                int64_t lddyk, int64_t hddyk, const void *q, int64_t ldq,
                                int64_t hdq, const void *k, int64_t ldk, int64_t hdk,
                                const void *wq, const void *wk, const float *freq,
                                const int32_t *pos, void *dq, int64_t lddq, int64_t hddq, void *dk,
                                int64_t lddk, int64_t hddk, float *dwq, float *dwk, void *work,
                                int64_t tokens, int64_t hq, int64_t hk, int64_t dim, int64_t rot,
                                float eps, int flags, int elem, void *hip_stream) {
  const Sizes s{tokens, hq, hk, dim, rot, eps, flags, elem};
  int rc = check_sizes(s);
  if (rc != TCU_OK) return rc;
  QkNormArgs a{};
  a.dy[0] = Heads{dyq, lddyq, hddyq};
  a.dy[1] = Heads{dyk, lddyk, hddyk};
  a.x[0] = Heads{q, ldq, hdq};
  a.x[1] = Heads{k, ldk, hdk};
  a.y[0] = Heads{dq, lddq, hddq};
  a.y[1] = Heads{dk, lddk, hddk};
  const bool heads = hq + hk > 0, any = tokens > 0 && heads;
  const int64_t es = elem_size(elem);
  const Operand ops[] = {
      heads_view(a.y[0], hq, s, true), heads_view(a.y[1], hk, s, true),
      vec(dwq, hq > 0 ? dim : 0, 4, 4, true), vec(dwk, hk > 0 ? dim : 0, 4, 4, true),
      vec(work, any ? tcu_qk_norm_grad_work(tokens, hq, hk, dim) : 0, 1, 16, true),
      heads_view(a.x[0], hq, s), heads_view(a.x[1], hk, s), heads_view(a.dy[0], hq, s),
      heads_view(a.dy[1], hk, s), vec(wq, any && hq > 0 ? dim : 0, es, 16),
      vec(wk, any && hk > 0 ? dim : 0, es, 16), vec(freq, any ? rot / 2 : 0, 4, 4),
      vec(pos, any && rot > 0 ? tokens : 0, 4, 4)};
  rc = check_operands(ops, {{same(a.y[0], a.x[0]) ? 0 : -1, 5}, {same(a.y[1], a.x[1]) ? 1 : -1, 6},
                            {same(a.y[0], a.dy[0]) ? 0 : -1, 7},
                            {same(a.y[1], a.dy[1]) ? 1 : -1, 8}});
  if (rc != TCU_OK) return rc;
  if (!heads) return TCU_OK;
  int num_cus = 0;
  rc = device_ready(&num_cus);
  if (rc != TCU_OK) return rc;
  rc = check_device(ops);
  if (rc != TCU_OK) return rc;
  a.w[0] = wq;
  a.w[1] = wk;
  a.dw[0] = hq > 0 ? dwq : nullptr;
  a.dw[1] = hk > 0 ? dwk : nullptr;
  a.parts = (float *)work;
  a.freq = freq;
  a.pos = pos;
  a.tokens = tokens;
  a.heads[0] = (int)hq;
  a.heads[1] = (int)hk;
  a.dim = (int)dim;
  a.rot = (int)rot;
  a.eps = eps;
  a.adjacent = (flags & TCU_ROPE_ADJACENT) != 0;
  return launch_qk_norm_grad(elem, a, (hipStream_t)hip_stream, num_cus) == hipSuccess
             ? TCU_OK
             : TCU_ERR_HIP;
}
