// Host runtime of the routing rules and the layer norm behind include/moe.h:
// argument checks, the router handle and its workspace.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <mutex>
#include <new>
#include <set>

#include "moe.h"
#include "moe_internal.h"

namespace moe {
void set_last_error(const char* msg);  // moe_api.cpp
}

using namespace moe;

struct moe_router {
  RouterParams p;
  int32_t max_tokens = 0, device = -1;
  bool backward = false;
  int users = 0;            // layers that route by it
  void* arena = nullptr;
};

namespace {

std::mutex g_router_mu;
std::set<moe_router*> g_router_live;

moe_status rfail(moe_status st, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  set_last_error(buf);
  // reported here, not by the check of a later launch that succeeds
  if (st == MOE_ENOMEM || st == MOE_EHIP) (void)hipGetLastError();
  return st;
}

moe_status rhfail(hipError_t e, const char* what) {
  return rfail(MOE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

bool aligned(const void* p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }

bool live(moe_router* r) {
  std::lock_guard<std::mutex> g(g_router_mu);
  return r && g_router_live.count(r) != 0;
}

moe_status check_desc(const moe_router_desc* d) {
  if (!d) return rfail(MOE_EINVAL, "desc is NULL");
  if (d->d_model <= 0 || d->d_model % 64 || d->d_model > 16384)
    return rfail(MOE_EINVAL, "d_model must be a positive multiple of 64, <= 16384 (got %d)", d->d_model);
  if (d->n_experts < 1 || d->n_experts > kRouterMaxExperts)
    return rfail(MOE_EINVAL, "n_experts must be in [1, %d] (got %d)", kRouterMaxExperts, d->n_experts);
  if (d->n_groups < 1 || d->n_groups > kRouterMaxGroups || d->n_experts % d->n_groups)
    return rfail(MOE_EINVAL, "n_groups must be in [1, %d] and divide n_experts (got %d of %d)",
                 kRouterMaxGroups, d->n_groups, d->n_experts);
  if (d->top_groups < 1 || d->top_groups > d->n_groups)
    return rfail(MOE_EINVAL, "top_groups must be in [1, n_groups] (got %d)", d->top_groups);
  const int held = d->top_groups * (d->n_experts / d->n_groups);
  if (d->top_k < 1 || d->top_k > kRouterMaxTopK || d->top_k > held)
    return rfail(MOE_EINVAL, "top_k must be in [1, min(%d, the %d experts of top_groups groups)] (got %d)",
                 kRouterMaxTopK, held, d->top_k);
  if (d->group_best != 1 && d->group_best != 2)
    return rfail(MOE_EINVAL, "group_best must be 1 or 2 (got %d)", d->group_best);
  if (d->max_tokens < 1 || d->max_tokens > 65536)
    return rfail(MOE_EINVAL, "max_tokens must be in [1, 65536] (got %d)", d->max_tokens);
  if (d->type != MOE_F16 && d->type != MOE_BF16) return rfail(MOE_EINVAL, "unknown type %d", d->type);
  if (d->score != MOE_SCORE_SOFTMAX && d->score != MOE_SCORE_SIGMOID)
    return rfail(MOE_EINVAL, "unknown score %d", d->score);
  if (d->renormalize != 0 && d->renormalize != 1)
    return rfail(MOE_EINVAL, "renormalize must be 0 or 1 (got %d)", d->renormalize);
  if (!(d->scale > 0.0f) || !std::isfinite(d->scale))
    return rfail(MOE_EINVAL, "scale must be finite and > 0");
  if (d->flags & ~(uint32_t)MOE_ROUTER_BACKWARD) return rfail(MOE_EINVAL, "unknown flags");
  return MOE_OK;
}

moe_status check_norm(int32_t type, int32_t n_tokens, int32_t d_model, float eps) {
  if (type != MOE_F16 && type != MOE_BF16) return rfail(MOE_EINVAL, "unknown type %d", type);
  // (a launch has less than 2^32 threads, and a row up to 1024)
  if (n_tokens < 1 || n_tokens > 1 << 21)
    return rfail(MOE_EINVAL, "n_tokens must be in [1, 2097152] (got %d)", n_tokens);
  if (d_model <= 0 || d_model % 64 || d_model > 16384)
    return rfail(MOE_EINVAL, "d_model must be a positive multiple of 64, <= 16384 (got %d)", d_model);
  if (!(eps >= 0.0f)) return rfail(MOE_EINVAL, "eps must be >= 0");
  return MOE_OK;
}

}  // namespace

namespace moe {

bool router_use(moe_router* r, RouterUse* out) {
  std::lock_guard<std::mutex> g(g_router_mu);
  if (!r || !g_router_live.count(r)) return false;
  out->p = r->p;
  out->max_tokens = r->max_tokens;
  out->device = r->device;
  return true;
}

bool router_hold(moe_router* r, int by) {
  std::lock_guard<std::mutex> g(g_router_mu);
  if (!r || !g_router_live.count(r)) return false;
  r->users += by;
  return true;
}

}  // namespace moe

extern "C" {

moe_status moe_router_init(const moe_router_desc* desc, const void* w_router, const float* bias,
                           moe_router_t* out) {
  set_last_error("");
  if (!out) return rfail(MOE_EINVAL, "out is NULL");
  *out = nullptr;
  const moe_status st = check_desc(desc);
  if (st != MOE_OK) return st;
  if (!w_router) return rfail(MOE_EINVAL, "w_router must not be NULL");
  if (!aligned(w_router, 16)) return rfail(MOE_EINVAL, "w_router must be 16-byte aligned");
  if (!aligned(bias, 4)) return rfail(MOE_EINVAL, "bias must be 4-byte aligned");
  moe_router* r = new (std::nothrow) moe_router();
  if (!r) return rfail(MOE_ENOMEM, "host allocation failed");
  hipError_t he = hipGetDevice(&r->device);
  if (he != hipSuccess) {
    delete r;
    return rhfail(he, "hipGetDevice");
  }
  r->max_tokens = desc->max_tokens;
  r->backward = (desc->flags & MOE_ROUTER_BACKWARD) != 0;
  RouterParams& p = r->p;
  p.wg = w_router;
  p.bias = bias;
  p.d = desc->d_model;
  p.E = desc->n_experts;
  p.K = desc->top_k;
  p.type = desc->type;
  p.score = desc->score;
  p.n_groups = desc->n_groups;
  const int32_t size = desc->n_experts / desc->n_groups;
  p.size_inv = ((1 << 20) + size - 1) / size;
  p.top_groups = desc->top_groups;
  p.group_best = desc->group_best;
  p.renorm = desc->renormalize;
  p.scale = desc->scale;
  auto al = [](size_t b) { return (b + 255) & ~(size_t)255; };
  const size_t rows = (size_t)desc->max_tokens * desc->n_experts;
  size_t off = 0;
  const size_t o_lg = off; off += al(rows * sizeof(float));
  const size_t o_xn = off; off += al(sizeof(float) * desc->max_tokens);
  const size_t o_wn = off; off += al(sizeof(float) * desc->n_experts);
  const size_t o_open = off; off += al(sizeof(int32_t) * (1 + (size_t)desc->max_tokens));
  const size_t o_grad = off;
  if (r->backward) off += router_backward_bytes(p.type, desc->max_tokens, p.d, p.E);
  he = hipMalloc(&r->arena, off);
  if (he != hipSuccess) {
    delete r;
    return rfail(MOE_ENOMEM, "hipMalloc of %zu router bytes failed: %s", off, hipGetErrorString(he));
  }
  char* base = static_cast<char*>(r->arena);
  p.logits = reinterpret_cast<float*>(base + o_lg);
  p.x_norm = reinterpret_cast<float*>(base + o_xn);
  p.w_norm = reinterpret_cast<float*>(base + o_wn);
  p.open = reinterpret_cast<int32_t*>(base + o_open);
  p.grad_ws = r->backward ? base + o_grad : nullptr;
  try {
    std::lock_guard<std::mutex> g(g_router_mu);
    g_router_live.insert(r);
  } catch (...) {
    (void)hipFree(r->arena);
    delete r;
    return rfail(MOE_ENOMEM, "host allocation failed");
  }
  *out = r;
  return MOE_OK;
}

moe_status moe_route(moe_router_t r, int32_t n_tokens, const void* x, int32_t* topk_idx,
                     float* topk_w, float* logits, int32_t* expert_count, void* stream) {
  set_last_error("");
  if (!live(r)) return rfail(MOE_ESTATE, "invalid or destroyed router handle");
  if (n_tokens < 1 || n_tokens > r->max_tokens)
    return rfail(MOE_EINVAL, "n_tokens must be in [1, %d] (got %d)", r->max_tokens, n_tokens);
  if (!x || !topk_idx || !topk_w) return rfail(MOE_EINVAL, "x, topk_idx and topk_w must not be NULL");
  if (!aligned(x, 16) || !aligned(logits, 16)) return rfail(MOE_EINVAL, "x and logits must be 16-byte aligned");
  if (!aligned(topk_idx, 4) || !aligned(topk_w, 4) || !aligned(expert_count, 4))
    return rfail(MOE_EINVAL, "topk_idx, topk_w and expert_count must be 4-byte aligned");
  hipError_t he = hipSetDevice(r->device);
  if (he != hipSuccess) return rhfail(he, "hipSetDevice");
  RouterOut o;
  o.idx = topk_idx;
  o.w = topk_w;
  o.logits = logits;
  o.count = expert_count;
  he = launch_router(r->p, n_tokens, x, o, static_cast<hipStream_t>(stream));
  if (he != hipSuccess) return rhfail(he, "router kernel launch");
  return MOE_OK;
}

moe_status moe_route_backward(moe_router_t r, int32_t n_tokens, const void* x, const float* logits,
                              const int32_t* topk_idx, const float* d_topk_w,
                              const float* d_logits, void* d_x, float* d_w_router, void* stream) {
  set_last_error("");
  if (!live(r)) return rfail(MOE_ESTATE, "invalid or destroyed router handle");
  if (!r->backward) return rfail(MOE_ESTATE, "the router was created without MOE_ROUTER_BACKWARD");
  if (n_tokens < 1 || n_tokens > r->max_tokens)
    return rfail(MOE_EINVAL, "n_tokens must be in [1, %d] (got %d)", r->max_tokens, n_tokens);
  if (!x || !logits || !topk_idx || !d_topk_w)
    return rfail(MOE_EINVAL, "x, logits, topk_idx and d_topk_w must not be NULL");
  if (!d_x && !d_w_router) return rfail(MOE_EINVAL, "d_x and d_w_router are both NULL");
  if (!aligned(x, 16) || !aligned(logits, 16) || !aligned(d_logits, 16) || !aligned(d_x, 16) ||
      !aligned(d_w_router, 16))
    return rfail(MOE_EINVAL, "x, logits, d_logits, d_x and d_w_router must be 16-byte aligned");
  if (!aligned(topk_idx, 4) || !aligned(d_topk_w, 4))
    return rfail(MOE_EINVAL, "topk_idx and d_topk_w must be 4-byte aligned");
  hipError_t he = hipSetDevice(r->device);
  if (he != hipSuccess) return rhfail(he, "hipSetDevice");
  he = launch_router_backward(r->p, n_tokens, x, logits, topk_idx, d_topk_w, d_logits, d_x,
                              d_w_router, static_cast<hipStream_t>(stream));
  if (he != hipSuccess) return rhfail(he, "router backward launch");
  return MOE_OK;
}

moe_status moe_router_destroy(moe_router_t r) {
  set_last_error("");
  if (!r) return rfail(MOE_EINVAL, "router is NULL");
  {
    std::lock_guard<std::mutex> g(g_router_mu);
    if (!g_router_live.count(r)) return rfail(MOE_ESTATE, "invalid or destroyed router handle");
    if (r->users > 0)
      return rfail(MOE_ESTATE, "%d layer(s) still route by this router", r->users);
    g_router_live.erase(r);
  }
  hipError_t he = hipSetDevice(r->device);
  if (he == hipSuccess) he = hipDeviceSynchronize();
  (void)hipFree(r->arena);
  delete r;
  if (he != hipSuccess) return rhfail(he, "destroy synchronize");
  return MOE_OK;
}

moe_status moe_layernorm(const float* h, const float* gain, const float* bias, void* x,
                         int32_t type, int32_t n_tokens, int32_t d_model, float eps,
                         void* stream) {
  set_last_error("");
  if (!h || !x) return rfail(MOE_EINVAL, "h and x must not be NULL");
  const moe_status st = check_norm(type, n_tokens, d_model, eps);
  if (st != MOE_OK) return st;
  if (!aligned(h, 16) || !aligned(x, 16) || !aligned(gain, 16) || !aligned(bias, 16))
    return rfail(MOE_EINVAL, "h, gain, bias and x must be 16-byte aligned");
  const hipError_t he = launch_layernorm(h, gain, bias, x, type, n_tokens, d_model, eps,
                                         static_cast<hipStream_t>(stream));
  if (he != hipSuccess) return rhfail(he, "layer norm launch");
  return MOE_OK;
}

moe_status moe_layernorm_workspace(int32_t n_tokens, int32_t d_model, int64_t* bytes) {
  set_last_error("");
  if (!bytes) return rfail(MOE_EINVAL, "bytes is NULL");
  *bytes = 0;
  const moe_status st = check_norm(MOE_F16, n_tokens, d_model, 0.0f);
  if (st != MOE_OK) return st;
  *bytes = (int64_t)layernorm_workspace(n_tokens, d_model);
  return MOE_OK;
}

moe_status moe_layernorm_backward(const void* d_x, int32_t type, const float* h,
                                  const float* gain, float eps, int32_t n_tokens,
                                  int32_t d_model, float* d_h, int32_t accumulate,
                                  float* d_gain, float* d_bias, void* workspace, void* stream) {
  set_last_error("");
  if (!d_x || !h || !d_h) return rfail(MOE_EINVAL, "d_x, h and d_h must not be NULL");
  const moe_status st = check_norm(type, n_tokens, d_model, eps);
  if (st != MOE_OK) return st;
  if ((d_gain || d_bias) && !workspace)
    return rfail(MOE_EINVAL, "d_gain and d_bias need a workspace");
  if (!aligned(d_x, 16) || !aligned(h, 16) || !aligned(gain, 16) || !aligned(d_h, 16) ||
      !aligned(d_gain, 16) || !aligned(d_bias, 16) || !aligned(workspace, 16))
    return rfail(MOE_EINVAL, "pointers must be 16-byte aligned");
  const hipError_t he = launch_layernorm_backward(d_x, type, h, gain, eps, n_tokens, d_model, d_h,
                                                  accumulate != 0, d_gain, d_bias, workspace,
                                                  static_cast<hipStream_t>(stream));
  if (he != hipSuccess) return rhfail(he, "layer norm backward launch");
  return MOE_OK;
}

}  // extern "C"
