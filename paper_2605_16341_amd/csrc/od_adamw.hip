// AdamW with decoupled weight decay over a list of tensors of any lengths: one elementwise pass,
//   m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2,   t = t + 1,
//   x = (1 - lr wd) x - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// HBM bound: g read, x, m and v read and written, 22 bytes an element in bf16 and 28 in fp32 (131 million bf16 elements 546 us,
// 5.29 TB/s; a copy of 4 GiB reaches 4.73).  The tensors' pointers
// travel in the launch's arguments, so a list of up to kAdamChunk tensors is one launch and needs no workspace.  t lives
// in device memory, where a captured graph finds it advanced at every replay: all workgroups read it, the last
// one of the last launch to finish adds one.
#include <hip/hip_runtime.h>

#include <cmath>
#include <memory>
#include <new>
#include <vector>

#include "../../include/orthdion.h"
#include "od_common.h"

// A launch has fewer than 2^32 threads.
constexpr int64_t kMostBlocks = (1 << 24) - 1;
constexpr int64_t kMostLength = (int64_t)1 << 35;

namespace od {

constexpr int kAdamChunk = 56;             // tensors of a launch: 56 bytes each, 3.2 of the 4 KB of its arguments
constexpr int kAdamThreads = 256;
constexpr int kAdamSpan = 4096;            // elements of a workgroup

struct AdamTensor {
  void* X;
  const void* G;
  float* M;
  float* V;
  int64_t n;
  float keep, step;                        // 1 - lr wd, lr
  int first;                               // first workgroup
  int vec;                                 // all four 16-byte aligned
};

struct AdamArgs {
  AdamTensor t[kAdamChunk];
  int count, blocks, last;
  int* counter;
  double beta1, beta2;
  float eps;
};

static_assert(sizeof(AdamTensor) == 56 && sizeof(AdamArgs) <= 4096, "arguments of a launch");

OD_DEV double power(double x, int n) {
  double r = 1.0;
  for (; n > 0; n >>= 1, x *= x)
    if (n & 1) r *= x;
  return r;
}

struct AdamCoef {                          // c1 and c2: 1 / (1 - b1^t) and the root of 1 / (1 - b2^t)
  float b1, a1, b2, a2, c1, c2, eps, keep, step;
};

OD_DEV float adam_one(float x, float g, float& m, float& v, const AdamCoef& k) {
  m = k.b1 * m + k.a1 * g;
  // factor by factor, so that only a v out of range overflows: g^2 does from 1.8e19 on, v / (1 - b2^t) is g^2 at first
  v = k.b2 * v + k.a2 * g * g;
  // rounded square root and quotient: the hardware's own take v or d below 2^-126 for zero, which with eps = 0 moved x to infinity
  const float d = __builtin_sqrtf(v) * k.c2 + k.eps;
  return k.keep * x - k.step * (m * k.c1 / d);
}

template <bool XBF, bool GBF>
__global__ __launch_bounds__(kAdamThreads) void k_adamw(AdamArgs a) {
  const int bid = blockIdx.x, tid = threadIdx.x;
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.t[mid].first <= bid) lo = mid;
    else hi = mid - 1;
  }
  const AdamTensor& t = a.t[lo];
  const int steps = a.counter[0] + 1;
  const AdamCoef k{(float)a.beta1, (float)(1.0 - a.beta1), (float)a.beta2, (float)(1.0 - a.beta2),
                   (float)(1.0 / (1.0 - power(a.beta1, steps))), (float)sqrt(1.0 / (1.0 - power(a.beta2, steps))), a.eps, t.keep, t.step};
  const int64_t begin = (int64_t)(bid - t.first) * kAdamSpan, end = min(t.n, begin + kAdamSpan);
  uint16_t* xh = reinterpret_cast<uint16_t*>(t.X);
  float* xf = reinterpret_cast<float*>(t.X);
  const uint16_t* gh = reinterpret_cast<const uint16_t*>(t.G);
  const float* gf = reinterpret_cast<const float*>(t.G);
  int64_t at = begin;
  if (t.vec) {
    for (int64_t i = begin + tid * 8; i + 8 <= end; i += kAdamThreads * 8) {
      float x[8], g[8], m[8], v[8];
      f32x4* mp = reinterpret_cast<f32x4*>(t.M + i);
      f32x4* vp = reinterpret_cast<f32x4*>(t.V + i);
      SrcF32::unpack8(SrcF32::Raw8{mp[0], mp[1]}, m);
      SrcF32::unpack8(SrcF32::Raw8{vp[0], vp[1]}, v);
      if constexpr (GBF) SrcBF16::unpack8(*reinterpret_cast<const u32x4*>(gh + i), g);
      else SrcF32::unpack8(SrcF32::Raw8{reinterpret_cast<const f32x4*>(gf + i)[0], reinterpret_cast<const f32x4*>(gf + i)[1]}, g);
      if constexpr (XBF) SrcBF16::unpack8(*reinterpret_cast<const u32x4*>(xh + i), x);
      else SrcF32::unpack8(SrcF32::Raw8{reinterpret_cast<const f32x4*>(xf + i)[0], reinterpret_cast<const f32x4*>(xf + i)[1]}, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = adam_one(x[e], g[e], m[e], v[e], k);
      mp[0] = f32x4{m[0], m[1], m[2], m[3]};
      mp[1] = f32x4{m[4], m[5], m[6], m[7]};
      vp[0] = f32x4{v[0], v[1], v[2], v[3]};
      vp[1] = f32x4{v[4], v[5], v[6], v[7]};
      if constexpr (XBF) {
        *reinterpret_cast<u32x4*>(xh + i) = u32x4{pack_bf16_rne(x[0], x[1]), pack_bf16_rne(x[2], x[3]), pack_bf16_rne(x[4], x[5]), pack_bf16_rne(x[6], x[7])};
      } else {
        reinterpret_cast<f32x4*>(xf + i)[0] = f32x4{x[0], x[1], x[2], x[3]};
        reinterpret_cast<f32x4*>(xf + i)[1] = f32x4{x[4], x[5], x[6], x[7]};
      }
    }
    at = begin + (end - begin) / 8 * 8;
  }
  for (int64_t i = at + tid; i < end; i += kAdamThreads) {
    float m = t.M[i], v = t.V[i];
    const float g = GBF ? bf16_bits_to_f32(gh[i]) : gf[i], x0 = XBF ? bf16_bits_to_f32(xh[i]) : xf[i];
    const float x = adam_one(x0, g, m, v, k);
    t.M[i] = m;
    t.V[i] = v;
    if constexpr (XBF) xh[i] = (uint16_t)pack_bf16_rne(x, 0.f);
    else xf[i] = x;
  }
  if (a.last) {
    __syncthreads();                       // every thread has read the counter
    if (tid == 0 && atomicAdd(a.counter + 1, 1) == a.blocks - 1) {
      a.counter[1] = 0;
      a.counter[0] = steps;
    }
  }
}

}  // namespace od

struct orthdion_adamw_ctx {
  std::vector<orthdion_adamw_desc> tensors;
  orthdion_adamw_config cfg;
};

template <class F>
static int no_throw(F&& body) {
  try {
    return body();
  } catch (const std::bad_alloc&) {
    return ORTHDION_E_NO_MEMORY;
  } catch (...) {
    return ORTHDION_E_INVALID_ARG;
  }
}

static int adamw_create(orthdion_adamw_handle* out, const orthdion_adamw_desc* tensors, int32_t count, const orthdion_adamw_config* cfg) {
  if (!tensors || !cfg) return ORTHDION_E_NULL_PTR;
  if (count < 1 || count > (1 << 20)) return ORTHDION_E_INVALID_ARG;
  if (cfg->x_dtype != ORTHDION_F32 && cfg->x_dtype != ORTHDION_BF16) return ORTHDION_E_INVALID_ARG;
  if (cfg->g_dtype != ORTHDION_F32 && cfg->g_dtype != ORTHDION_BF16) return ORTHDION_E_INVALID_ARG;
  if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0)) return ORTHDION_E_INVALID_ARG;
  if (!std::isfinite(cfg->lr) || !std::isfinite(cfg->eps) || cfg->eps < 0.f) return ORTHDION_E_INVALID_ARG;
  for (int i = 0; i < count; ++i) {
    if (tensors[i].length < 0 || tensors[i].length >= kMostLength) return ORTHDION_E_BAD_SHAPE;
    if (!std::isfinite(tensors[i].weight_decay) || !std::isfinite(tensors[i].lr_scale)) return ORTHDION_E_INVALID_ARG;
  }
  orthdion_adamw_ctx* h = new (std::nothrow) orthdion_adamw_ctx();
  if (!h) return ORTHDION_E_NO_MEMORY;
  *out = h;
  h->tensors.assign(tensors, tensors + count);
  h->cfg = *cfg;
  return ORTHDION_OK;
}

extern "C" int orthdion_adamw_create(orthdion_adamw_handle* out, const orthdion_adamw_desc* tensors, int32_t count,
                                     const orthdion_adamw_config* cfg) {
  if (!out) return ORTHDION_E_NULL_PTR;
  *out = nullptr;
  orthdion_adamw_handle h = nullptr;
  const int rc = no_throw([&] { return adamw_create(&h, tensors, count, cfg); });
  if (rc != ORTHDION_OK) {
    delete h;
    return rc;
  }
  *out = h;
  return ORTHDION_OK;
}

extern "C" int orthdion_adamw_set_lr(orthdion_adamw_handle h, float lr) {
  if (!h) return ORTHDION_E_NULL_PTR;
  if (!std::isfinite(lr)) return ORTHDION_E_INVALID_ARG;
  h->cfg.lr = lr;
  return ORTHDION_OK;
}

extern "C" int orthdion_adamw_step(orthdion_adamw_handle h, void* const* X, const void* const* G, float* const* M, float* const* V,
                                   int32_t* counter, void* stream) {
  using namespace od;
  if (!h || !X || !G || !M || !V || !counter) return ORTHDION_E_NULL_PTR;
  if (reinterpret_cast<uintptr_t>(counter) % 4) return ORTHDION_E_MISALIGNED;
  const int total = (int)h->tensors.size();
  const bool xbf = h->cfg.x_dtype == ORTHDION_BF16, gbf = h->cfg.g_dtype == ORTHDION_BF16;
  const size_t xe = xbf ? 2 : 4, ge = gbf ? 2 : 4;
  for (int i = 0; i < total; ++i) {
    if (h->tensors[i].length == 0) continue;                  // nothing behind its pointers
    if (!X[i] || !G[i] || !M[i] || !V[i]) return ORTHDION_E_NULL_PTR;
    if (reinterpret_cast<uintptr_t>(X[i]) % xe || reinterpret_cast<uintptr_t>(G[i]) % ge ||
        reinterpret_cast<uintptr_t>(M[i]) % 4 || reinterpret_cast<uintptr_t>(V[i]) % 4)
      return ORTHDION_E_MISALIGNED;
  }
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const std::unique_ptr<AdamArgs> a(new (std::nothrow) AdamArgs());
  if (!a) return ORTHDION_E_NO_MEMORY;
  a->counter = counter;
  a->beta1 = h->cfg.beta1;
  a->beta2 = h->cfg.beta2;
  a->eps = h->cfg.eps;
  auto flush = [&](bool last) {
    a->last = last ? 1 : 0;
    if (a->count == 0) {                                      // nothing but the counter
      a->t[0] = AdamTensor{};
      a->count = 1;
      a->blocks = 1;
    }
    if (xbf) gbf ? k_adamw<true, true><<<a->blocks, kAdamThreads, 0, st>>>(*a) : k_adamw<true, false><<<a->blocks, kAdamThreads, 0, st>>>(*a);
    else gbf ? k_adamw<false, true><<<a->blocks, kAdamThreads, 0, st>>>(*a) : k_adamw<false, false><<<a->blocks, kAdamThreads, 0, st>>>(*a);
    a->count = 0;
    a->blocks = 0;
    return hipGetLastError();
  };
  for (int i = 0; i < total; ++i) {
    const orthdion_adamw_desc& d = h->tensors[i];
    if (d.length == 0) continue;
    // the workgroups of one tensor always fit a launch
    const int64_t need = (d.length + kAdamSpan - 1) / kAdamSpan;
    if (a->count == kAdamChunk || a->blocks + need > kMostBlocks)
      if (flush(false) != hipSuccess) return ORTHDION_E_HIP;
    AdamTensor& t = a->t[a->count++];
    const uintptr_t bits = reinterpret_cast<uintptr_t>(X[i]) | reinterpret_cast<uintptr_t>(G[i]) | reinterpret_cast<uintptr_t>(M[i]) | reinterpret_cast<uintptr_t>(V[i]);
    const double lr = (double)h->cfg.lr * (double)d.lr_scale;
    t = AdamTensor{X[i], G[i], M[i], V[i], d.length, (float)(1.0 - lr * (double)d.weight_decay), (float)lr, a->blocks, (bits & 15) == 0};
    a->blocks += (int)need;
  }
  return flush(true) == hipSuccess ? ORTHDION_OK : ORTHDION_E_HIP;
}

extern "C" int orthdion_adamw_destroy(orthdion_adamw_handle h) {
  if (!h) return ORTHDION_E_NULL_PTR;
  delete h;
  return ORTHDION_OK;
}
