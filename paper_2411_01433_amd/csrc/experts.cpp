// Host runtime of the products grouped by expert, the MXFP4 quantiser and the
// gradient lists behind include/moe.h: argument checks, the list handle.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <mutex>
#include <new>
#include <set>
#include <vector>

#include "moe.h"
#include "moe_internal.h"

namespace moe {
void set_last_error(const char* msg);  // moe_api.cpp
}

using namespace moe;

struct moe_gradients {
  GradList list;
  int32_t device = -1;
  void* arena = nullptr;
};

namespace {

std::mutex g_grad_mu;
std::set<moe_gradients*> g_grad_live;

moe_status efail(moe_status st, const char* fmt, ...) {
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

moe_status ehfail(hipError_t e, const char* what) {
  return efail(MOE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

bool aligned(const void* p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }

bool live(moe_gradients* g) {
  std::lock_guard<std::mutex> lock(g_grad_mu);
  return g && g_grad_live.count(g) != 0;
}

moe_status check_grouped(const int32_t* count, int32_t type, int32_t n_rows, int32_t d_in,
                         int32_t d_out, int32_t n_experts) {
  if (type != MOE_F16 && type != MOE_BF16) return efail(MOE_EINVAL, "unknown type %d", type);
  if (n_rows < 0 || n_rows > kGroupedMaxRows)
    return efail(MOE_EINVAL, "n_rows must be in [0, %d] (got %d)", kGroupedMaxRows, n_rows);
  if (d_in <= 0 || d_in % 64 || d_in > 65536 || d_out <= 0 || d_out % 64 || d_out > 65536)
    return efail(MOE_EINVAL, "d_in and d_out must be positive multiples of 64, <= 65536 (got %d, %d)",
                 d_in, d_out);
  if (n_experts < 1 || n_experts > kRouterMaxExperts)
    return efail(MOE_EINVAL, "n_experts must be in [1, %d] (got %d)", kRouterMaxExperts, n_experts);
  if (!count && n_experts != 1)
    return efail(MOE_EINVAL, "%d experts need expert_count", n_experts);
  if (!aligned(count, 4)) return efail(MOE_EINVAL, "expert_count must be 4-byte aligned");
  return MOE_OK;
}

int64_t type_size(int32_t type) { return type == MOE_F32 ? 4 : 2; }

}  // namespace

extern "C" {

moe_status moe_grouped_product(const void* x, const void* w, const int32_t* expert_count, void* y,
                               int32_t type, int32_t n_rows, int32_t d_in, int32_t d_out,
                               int32_t n_experts, void* stream) {
  set_last_error("");
  const moe_status st = check_grouped(expert_count, type, n_rows, d_in, d_out, n_experts);
  if (st != MOE_OK) return st;
  if (!w || (n_rows > 0 && (!x || !y))) return efail(MOE_EINVAL, "x, w and y must not be NULL");
  if (!aligned(x, 16) || !aligned(w, 16) || !aligned(y, 16))
    return efail(MOE_EINVAL, "x, w and y must be 16-byte aligned");
  if (n_rows == 0) return MOE_OK;
  const Grouped g = {expert_count, type, n_rows, d_in, d_out, n_experts};
  const hipError_t he = launch_grouped_product(g, x, w, y, static_cast<hipStream_t>(stream));
  if (he != hipSuccess) return ehfail(he, "grouped product launch");
  return MOE_OK;
}

moe_status moe_grouped_product_backward(const void* d_y, const void* x, const void* w,
                                        const int32_t* expert_count, void* d_x, float* d_w,
                                        int32_t accumulate, int32_t type, int32_t n_rows,
                                        int32_t d_in, int32_t d_out, int32_t n_experts,
                                        void* stream) {
  set_last_error("");
  const moe_status st = check_grouped(expert_count, type, n_rows, d_in, d_out, n_experts);
  if (st != MOE_OK) return st;
  // (a tensor of no rows may be NULL: that says nothing about what is asked for)
  if (!d_x && !d_w && n_rows > 0) return efail(MOE_EINVAL, "d_x and d_w are both NULL");
  if (n_rows > 0 && !d_y) return efail(MOE_EINVAL, "d_y must not be NULL");
  if (d_x && !w) return efail(MOE_EINVAL, "d_x needs w");
  if (d_w && n_rows > 0 && !x) return efail(MOE_EINVAL, "d_w needs x");
  if (!aligned(d_y, 16) || !aligned(x, 16) || !aligned(w, 16) || !aligned(d_x, 16) ||
      !aligned(d_w, 16))
    return efail(MOE_EINVAL, "d_y, x, w, d_x and d_w must be 16-byte aligned");
  const Grouped g = {expert_count, type, n_rows, d_in, d_out, n_experts};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (d_x && n_rows > 0) {
    const hipError_t he = launch_grouped_dx(g, d_y, w, d_x, s);
    if (he != hipSuccess) return ehfail(he, "grouped product backward launch");
  }
  // (without rows: zeros)
  if (d_w && (n_rows > 0 || !accumulate)) {
    const hipError_t he = launch_grouped_dw(g, d_y, x, d_w, accumulate != 0, s);
    if (he != hipSuccess) return ehfail(he, "grouped product backward launch");
  }
  return MOE_OK;
}

moe_status moe_mx_quantize(const void* v, int32_t type, int64_t rows, int64_t cols, void* codes,
                           void* scales, void* values, void* stream) {
  set_last_error("");
  if (type != MOE_F16 && type != MOE_BF16) return efail(MOE_EINVAL, "unknown type %d", type);
  if (cols <= 0 || cols % 64 || cols > 65536)
    return efail(MOE_EINVAL, "cols must be a positive multiple of 64, <= 65536 (got %lld)",
                 (long long)cols);
  if (rows < 0 || rows > INT32_MAX || rows * cols >= (int64_t)1 << 36)
    return efail(MOE_EINVAL, "rows must be in [0, 2^31) and rows * cols < 2^36 (got %lld)",
                 (long long)rows);
  if (rows > 0 && (!v || !codes || !scales))
    return efail(MOE_EINVAL, "v, codes and scales must not be NULL");
  if (!aligned(v, 16) || !aligned(codes, 16) || !aligned(values, 16))
    return efail(MOE_EINVAL, "v, codes and values must be 16-byte aligned");
  if (!aligned(scales, 2)) return efail(MOE_EINVAL, "scales must be 2-byte aligned");
  const hipError_t he = launch_mx_quantize(v, type, rows, cols, static_cast<uint8_t*>(codes),
                                           static_cast<uint8_t*>(scales), values,
                                           static_cast<hipStream_t>(stream));
  if (he != hipSuccess) return ehfail(he, "MX quantiser launch");
  return MOE_OK;
}

moe_status moe_mx_product(const void* x, const void* x_scales, const void* w_codes,
                          const void* w_scales, const int32_t* expert_count, void* y, int32_t type,
                          int32_t n_rows, int32_t d_in, int32_t d_out, int32_t n_experts,
                          void* stream) {
  set_last_error("");
  const moe_status st = check_grouped(expert_count, type, n_rows, d_in, d_out, n_experts);
  if (st != MOE_OK) return st;
  if (!w_codes || !w_scales || (n_rows > 0 && (!x || !y)))
    return efail(MOE_EINVAL, "x, w_codes, w_scales and y must not be NULL");
  if (!aligned(x, 16) || !aligned(w_codes, 16) || !aligned(y, 16))
    return efail(MOE_EINVAL, "x, w_codes and y must be 16-byte aligned");
  if (!aligned(x_scales, 4) || !aligned(w_scales, 4))
    return efail(MOE_EINVAL, "scales must be 4-byte aligned");
  if (n_rows == 0) return MOE_OK;
  const Grouped g = {expert_count, type, n_rows, d_in, d_out, n_experts};
  const hipError_t he = launch_mx_product(g, x, static_cast<const uint8_t*>(x_scales),
                                          static_cast<const uint8_t*>(w_codes),
                                          static_cast<const uint8_t*>(w_scales), y,
                                          static_cast<hipStream_t>(stream));
  if (he != hipSuccess) return ehfail(he, "MX product launch");
  return MOE_OK;
}

moe_status moe_gradients_init(int32_t n, const void* const* grads, void* const* outs,
                              const int64_t* sizes, const int32_t* types, void* stream,
                              moe_gradients_t* out) {
  set_last_error("");
  if (!out) return efail(MOE_EINVAL, "out is NULL");
  *out = nullptr;
  if (n < 1 || n > 65536) return efail(MOE_EINVAL, "n must be in [1, 65536] (got %d)", n);
  if (!grads || !sizes || !types) return efail(MOE_EINVAL, "grads, sizes and types must not be NULL");
  moe_gradients* h = nullptr;
  try {
    struct Span {
      uintptr_t at;
      int64_t bytes;
    };
    std::vector<Span> spans;
    std::vector<GradPiece> pieces;
    int64_t total = 0;
    for (int32_t i = 0; i < n; ++i) {
      if (types[i] != MOE_F16 && types[i] != MOE_BF16 && types[i] != MOE_F32)
        return efail(MOE_EINVAL, "tensor %d: unknown type %d", i, types[i]);
      if (sizes[i] < 0 || sizes[i] >= (int64_t)1 << 38)
        return efail(MOE_EINVAL, "tensor %d: size must be in [0, 2^38) (got %lld)", i,
                     (long long)sizes[i]);
      if (sizes[i] == 0) continue;
      total += sizes[i];
      if (total >= (int64_t)1 << 38) return efail(MOE_EINVAL, "the sizes sum to 2^38 or more");
      const int64_t es = type_size(types[i]);
      const char* in = static_cast<const char*>(grads[i]);
      char* to = outs ? static_cast<char*>(outs[i]) : const_cast<char*>(in);
      if (!in || !to) return efail(MOE_EINVAL, "tensor %d is NULL", i);
      if (!aligned(in, (unsigned)es) || !aligned(to, (unsigned)es))
        return efail(MOE_EINVAL, "tensor %d must be aligned to its elements", i);
      spans.push_back({(uintptr_t)in, sizes[i] * es});
      if (to != in) spans.push_back({(uintptr_t)to, sizes[i] * es});
      const int64_t per = kPieceBytes / es;
      for (int64_t at = 0; at < sizes[i]; at += per)
        pieces.push_back({in + at * es, to + at * es, (int32_t)std::min(per, sizes[i] - at), types[i]});
    }
    if (pieces.empty()) pieces.push_back({nullptr, nullptr, 0, MOE_F32});  // nothing: norm 0
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.at < b.at; });
    for (size_t i = 1; i < spans.size(); ++i)
      if (spans[i].at - spans[i - 1].at < (uintptr_t)spans[i - 1].bytes)
        return efail(MOE_EINVAL, "two tensors overlap");
    h = new moe_gradients();
    hipError_t he = hipGetDevice(&h->device);
    if (he != hipSuccess) {
      delete h;
      return ehfail(he, "hipGetDevice");
    }
    auto al = [](size_t b) { return (b + 255) & ~(size_t)255; };
    const size_t count = pieces.size();
    const size_t o_sums = al(count * sizeof(GradPiece)), o_done = o_sums + al(kGradBlocks * sizeof(double));
    he = hipMalloc(&h->arena, o_done + 256);
    if (he != hipSuccess) {
      delete h;
      return efail(MOE_ENOMEM, "hipMalloc of %zu list bytes failed: %s", o_done + 256,
                   hipGetErrorString(he));
    }
    char* base = static_cast<char*>(h->arena);
    h->list = {reinterpret_cast<const GradPiece*>(base), reinterpret_cast<double*>(base + o_sums),
               reinterpret_cast<unsigned*>(base + o_done), (int32_t)count,
               (int32_t)std::min<size_t>(count, kGradBlocks)};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    he = hipMemcpyAsync(base, pieces.data(), count * sizeof(GradPiece), hipMemcpyHostToDevice, s);
    const uint32_t zero = 0;
    if (he == hipSuccess)
      he = hipMemcpyAsync(base + o_done, &zero, sizeof zero, hipMemcpyHostToDevice, s);
    const hipError_t hs = hipStreamSynchronize(s);  // (also where a copy failed: they read host memory)
    if (he == hipSuccess) he = hs;
    if (he != hipSuccess) {
      (void)hipFree(h->arena);
      delete h;
      return ehfail(he, "copy of the list");
    }
    std::lock_guard<std::mutex> lock(g_grad_mu);
    g_grad_live.insert(h);
  } catch (...) {
    if (h) {
      (void)hipFree(h->arena);
      delete h;
    }
    return efail(MOE_ENOMEM, "host allocation failed");
  }
  *out = h;
  return MOE_OK;
}

// After the checks: the handle's device, and what a launch answered.
static moe_status on_device(moe_gradients_t g) {
  const hipError_t he = hipSetDevice(g->device);
  return he == hipSuccess ? MOE_OK : ehfail(he, "hipSetDevice");
}
static moe_status launched(hipError_t he) {
  return he == hipSuccess ? MOE_OK : ehfail(he, "gradient kernel launch");
}

static moe_status check_gradients(moe_gradients_t g, float max_norm, const float* norm) {
  set_last_error("");
  if (!live(g)) return efail(MOE_ESTATE, "invalid or destroyed gradients handle");
  if (!norm) return efail(MOE_EINVAL, "norm is NULL");
  if (!aligned(norm, 4)) return efail(MOE_EINVAL, "norm must be 4-byte aligned");
  if (!(max_norm > 0.0f) || !std::isfinite(max_norm))
    return efail(MOE_EINVAL, "max_norm must be finite and > 0");
  return MOE_OK;
}

moe_status moe_gradients_norm(moe_gradients_t g, float* norm, void* stream) {
  moe_status st = check_gradients(g, 1.0f, norm);
  if (st == MOE_OK) st = on_device(g);
  return st != MOE_OK ? st : launched(launch_gradients_norm(g->list, norm, static_cast<hipStream_t>(stream)));
}

moe_status moe_gradients_scale(moe_gradients_t g, float max_norm, const float* norm, void* stream) {
  moe_status st = check_gradients(g, max_norm, norm);
  if (st == MOE_OK) st = on_device(g);
  return st != MOE_OK ? st
                      : launched(launch_gradients_scale(g->list, max_norm, norm, static_cast<hipStream_t>(stream)));
}

moe_status moe_gradients_clip(moe_gradients_t g, float max_norm, float* norm, void* stream) {
  moe_status st = check_gradients(g, max_norm, norm);
  if (st == MOE_OK) st = on_device(g);
  return st != MOE_OK ? st
                      : launched(launch_gradients_clip(g->list, max_norm, norm, static_cast<hipStream_t>(stream)));
}

moe_status moe_gradients_destroy(moe_gradients_t g) {
  set_last_error("");
  if (!g) return efail(MOE_EINVAL, "gradients is NULL");
  {
    std::lock_guard<std::mutex> lock(g_grad_mu);
    if (!g_grad_live.count(g)) return efail(MOE_ESTATE, "invalid or destroyed gradients handle");
    g_grad_live.erase(g);
  }
  hipError_t he = hipSetDevice(g->device);
  if (he == hipSuccess) he = hipDeviceSynchronize();
  (void)hipFree(g->arena);
  delete g;
  if (he != hipSuccess) return ehfail(he, "destroy synchronize");
  return MOE_OK;
}

}  // extern "C"
