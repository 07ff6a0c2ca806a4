// Host side of Muon's C ABI: argument checks, classes and clusters of matrices, the plan of the workspace, the scales
// of the fp16 operands, and the kernel sequence of a call.  No device memory is allocated here.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>
#include <vector>

#include "../../include/orthdion.h"
#include "od_muon.h"

namespace {

using od::MuonEntry;
using od::MuonMat;
using od::MuonTables;
using od::NsArgs;
using od::NsClass;

constexpr size_t kAlign = 256;
constexpr int64_t kMaxDim = 1 << 22;       // 32-bit offsets of the operand loads: 256 rows of 2^22 fp16 words
// Matrices step together (a cluster: every kernel of the iteration is one launch over it) up to this many elements; the
// next cluster reuses the workspace.
constexpr int64_t kClusterElements = (int64_t)1 << 28;
constexpr int64_t kPartElements = 16384;   // elements behind one partial sum of squares

size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
int up64(int64_t v) { return (int)((v + 63) / 64 * 64); }
// rows a multiple of 2 KB apart would put the rows of a tile on few memory channels
int pitch(int64_t v) { return up64(v) % 1024 == 0 ? up64(v) + 64 : up64(v); }

struct Cluster {
  NsArgs args;                             // `first` is left to the launchers, base to the call
  std::vector<int64_t> offset;             // bytes of the classes' slices behind the cluster's start
  int mat0, count;                         // rows of the matrix tables
};

struct Iteration {
  float a, b, c;
  int exp_y, exp_s, exp_p, exp_out;        // powers of two of the stored words: Y read, S, P, Y written
};

// power of two that brings values up to `bound` to 2^13 at most, three bits below the end of fp16's range
int exponent_for(double bound) { return 13 - (int)std::ceil(std::log2(bound)); }

}  // namespace

struct orthdion_muon_ctx {
  std::vector<orthdion_muon_matdesc> mats;
  orthdion_muon_config cfg;
  int parts;
  std::vector<Iteration> iterations;
  std::vector<int> order;                  // table row -> matrix
  std::vector<MuonMat> table;              // by row
  std::vector<Cluster> clusters;
  size_t off_entries, off_mats, off_partials, off_info, off_slices, ws_bytes;
  const void* last_ws = nullptr;
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

// Powers of two from bounds on the spectral norms, which bound every entry: sigma <= 1 at the start (Frobenius norm 1),
// then the largest |sigma (a + b sigma^2 + c sigma^4)| over the range before, with 2 % for the rounding of the iterate.
static int plan_iterations(orthdion_muon_ctx* h) {
  double top = 1.02;
  for (int k = 0; k < h->cfg.steps; ++k) {
    Iteration it;
    it.a = h->cfg.coeffs[3 * k]; it.b = h->cfg.coeffs[3 * k + 1]; it.c = h->cfg.coeffs[3 * k + 2];
    if (!std::isfinite(it.a) || !std::isfinite(it.b) || !std::isfinite(it.c)) return ORTHDION_E_INVALID_ARG;
    double poly = 0.0, next = 0.0;
    for (int i = 0; i <= 4096; ++i) {
      const double s = top * i / 4096, v = std::fabs(it.a + it.b * s * s + it.c * s * s * s * s);
      poly = std::max(poly, v);
      next = std::max(next, v * s);
    }
    if (!(poly <= 256.0) || !(next <= 32.0)) return ORTHDION_E_INVALID_ARG;
    poly = std::max(1.02 * poly, 1.0 / 256);
    next = std::max(1.02 * next, 1.0 / 256);
    it.exp_y = exponent_for(top);
    it.exp_s = exponent_for(top * top);
    it.exp_p = exponent_for(poly);
    it.exp_out = exponent_for(next);
    h->iterations.push_back(it);
    top = next;
  }
  return ORTHDION_OK;
}

static int check_muon_config(const orthdion_muon_config* c) {
  if (c->x_dtype != ORTHDION_F32 && c->x_dtype != ORTHDION_BF16) return ORTHDION_E_INVALID_ARG;
  if (c->g_dtype != ORTHDION_F32 && c->g_dtype != ORTHDION_BF16) return ORTHDION_E_INVALID_ARG;
  if (c->precision != ORTHDION_PREC_AUTO && c->precision != ORTHDION_PREC_FAST && c->precision != ORTHDION_PREC_EXACT)
    return ORTHDION_E_INVALID_ARG;
  if (c->nesterov != 0 && c->nesterov != 1) return ORTHDION_E_INVALID_ARG;
  if (c->steps < 1 || c->steps > ORTHDION_MUON_MAX_STEPS) return ORTHDION_E_INVALID_ARG;
  if (!std::isfinite(c->mu) || c->mu < 0.f || c->mu > 1.f) return ORTHDION_E_INVALID_ARG;
  if (!std::isfinite(c->lr) || !std::isfinite(c->weight_decay)) return ORTHDION_E_INVALID_ARG;
  if (!std::isfinite(c->eps) || c->eps < 0.f) return ORTHDION_E_INVALID_ARG;
  return ORTHDION_OK;
}

static int muon_create(orthdion_muon_handle* out, const orthdion_muon_matdesc* mats, int32_t nmat, const orthdion_muon_config* cfg) {
  if (!mats || !cfg) return ORTHDION_E_NULL_PTR;
  if (nmat < 1 || nmat > (1 << 20)) return ORTHDION_E_INVALID_ARG;
  int rc = check_muon_config(cfg);
  if (rc != ORTHDION_OK) return rc;
  for (int i = 0; i < nmat; ++i) {
    const orthdion_muon_matdesc& d = mats[i];
    if (d.m < 1 || d.n < 1 || d.m >= kMaxDim || d.n >= kMaxDim) return ORTHDION_E_BAD_SHAPE;
    if (d.ldx < d.n || d.ldg < d.n || d.ldm < d.n) return ORTHDION_E_BAD_SHAPE;
    if (!std::isfinite(d.scale)) return ORTHDION_E_INVALID_ARG;
  }
  orthdion_muon_ctx* h = new (std::nothrow) orthdion_muon_ctx();
  if (!h) return ORTHDION_E_NO_MEMORY;
  *out = h;                                // the caller frees it if anything below fails or throws
  h->mats.assign(mats, mats + nmat);
  h->cfg = *cfg;
  if ((rc = plan_iterations(h)) != ORTHDION_OK) return rc;
  const bool exact = cfg->precision == ORTHDION_PREC_EXACT ||
                     (cfg->precision == ORTHDION_PREC_AUTO && !(cfg->x_dtype == ORTHDION_BF16 && cfg->g_dtype == ORTHDION_BF16));
  h->parts = exact ? 2 : 1;

  // classes in order of first appearance
  struct Class { int p, q, tall; std::vector<int> members; };
  std::vector<Class> classes;
  for (int i = 0; i < nmat; ++i) {
    const int p = (int)std::min(mats[i].m, mats[i].n), q = (int)std::max(mats[i].m, mats[i].n), tall = mats[i].m > mats[i].n;
    size_t k = 0;
    while (k < classes.size() && !(classes[k].p == p && classes[k].q == q && classes[k].tall == tall)) ++k;
    if (k == classes.size()) classes.push_back(Class{p, q, tall, {}});
    classes[k].members.push_back(i);
  }
  // clusters
  int64_t held = 0;
  size_t slices = 0, most = 0;
  for (const Class& c : classes) {
    const int64_t elements = (int64_t)c.p * c.q;
    const int lp = pitch(c.p), lq = pitch(c.q);
    const int64_t stride = h->parts * 2 * (od::ns_y_plane(c.p, lq) + od::ns_s_plane(c.p, lp));
    for (size_t done = 0; done < c.members.size();) {
      if (h->clusters.empty() || held + elements > kClusterElements || h->clusters.back().args.nclass == od::kNsClasses) {
        h->clusters.push_back(Cluster{});
        h->clusters.back().mat0 = (int)h->order.size();
        held = 0;
        slices = 0;
      }
      Cluster& cl = h->clusters.back();
      const int64_t room = std::max((int64_t)1, (kClusterElements - held) / elements);
      // the workgroups of a launch are counted in 32 bits: a class of many matrices is 64 x 64 tiles at least
      const int take = (int)std::min<int64_t>({room, (int64_t)(c.members.size() - done), 1 << 20});
      NsClass& n = cl.args.c[cl.args.nclass++];
      n = NsClass{0, c.p, c.q, lp, lq, take, (int)h->order.size(), c.tall, nullptr, stride};
      cl.offset.push_back((int64_t)slices);
      slices = align_up(slices + (size_t)take * (size_t)stride * 2);
      most = std::max(most, slices);
      for (int k = 0; k < take; ++k) {
        const int i = c.members[done + k];
        const orthdion_muon_matdesc& d = mats[i];
        const int64_t parts = std::min<int64_t>({(d.m * d.n + kPartElements - 1) / kPartElements, od::kMuonParts, d.m});
        h->order.push_back(i);
        h->table.push_back(MuonMat{(int)d.m, (int)d.n, d.ldx, d.ldg, d.ldm, d.scale, (int)parts});
      }
      cl.count += take;
      held += take * elements;
      done += take;
    }
  }
  size_t off = 0;
  h->off_entries = off; off = align_up(off + (size_t)nmat * sizeof(MuonEntry));
  h->off_mats = off; off = align_up(off + (size_t)nmat * sizeof(MuonMat));
  h->off_partials = off; off = align_up(off + (size_t)nmat * od::kMuonParts * sizeof(double));
  h->off_info = off; off = align_up(off + (size_t)nmat * sizeof(int));
  h->off_slices = off;
  h->ws_bytes = off + most;
  return ORTHDION_OK;
}

#define OD_TRY(expr)                                   \
  do {                                                 \
    if ((expr) != hipSuccess) return ORTHDION_E_HIP;   \
  } while (0)

// X and M null: orthdion_muon_orthogonalise (A at G, O at X)
static int muon_run(orthdion_muon_handle h, void* const* X, const void* const* G, float* const* M, bool update, void* workspace,
                    size_t workspace_bytes, void* stream) {
  if (!h || !X || !G || (update && !M) || !workspace) return ORTHDION_E_NULL_PTR;
  if (workspace_bytes < h->ws_bytes) return ORTHDION_E_WORKSPACE_TOO_SMALL;
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign) return ORTHDION_E_MISALIGNED;
  const int nmat = (int)h->mats.size();
  const size_t xe = h->cfg.x_dtype == ORTHDION_BF16 ? 2 : 4, ge = h->cfg.g_dtype == ORTHDION_BF16 ? 2 : 4;
  for (int i = 0; i < nmat; ++i) {
    if (!X[i] || !G[i] || (update && !M[i])) return ORTHDION_E_NULL_PTR;
    if (reinterpret_cast<uintptr_t>(X[i]) % xe || reinterpret_cast<uintptr_t>(G[i]) % ge ||
        (update && reinterpret_cast<uintptr_t>(M[i]) % 4))
      return ORTHDION_E_MISALIGNED;
  }
  const std::unique_ptr<MuonEntry[]> entries(new (std::nothrow) MuonEntry[nmat]);
  if (!entries) return ORTHDION_E_NO_MEMORY;
  for (int r = 0; r < nmat; ++r) {
    const int i = h->order[r];
    entries[r] = MuonEntry{X[i], G[i], update ? M[i] : nullptr};
  }
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();                 // what an earlier, unrelated call left there
  char* ws = reinterpret_cast<char*>(workspace);
  h->last_ws = workspace;
  const MuonTables t{reinterpret_cast<MuonEntry*>(ws + h->off_entries), reinterpret_cast<const MuonMat*>(ws + h->off_mats),
                     reinterpret_cast<double*>(ws + h->off_partials), reinterpret_cast<int*>(ws + h->off_info)};
  const bool gbf = h->cfg.g_dtype == ORTHDION_BF16, xbf = h->cfg.x_dtype == ORTHDION_BF16, nesterov = h->cfg.nesterov != 0;
  const float keep = (float)(1.0 - (double)h->cfg.lr * (double)h->cfg.weight_decay);
  for (const Cluster& cl : h->clusters) {
    NsArgs a = cl.args;
    for (int k = 0; k < a.nclass; ++k) a.c[k].base = reinterpret_cast<uint16_t*>(ws + h->off_slices + cl.offset[k]);
    OD_TRY(od::launch_muon_begin(entries.get() + cl.mat0, h->table.data() + cl.mat0, cl.mat0, cl.count, t, h->cfg.mu, nesterov, gbf, st));
    OD_TRY(od::launch_muon_scale(a, t, h->cfg.mu, nesterov, gbf, h->parts, h->cfg.eps, std::ldexp(1.0, h->iterations[0].exp_y), st));
    const int steps = (int)h->iterations.size();
    for (int k = 0; k < steps; ++k) {
      const Iteration& it = h->iterations[k];
      const int src = k & 1;
      OD_TRY(od::launch_ns_gram(a, h->parts, src, std::ldexp(1.f, it.exp_s - 2 * it.exp_y), st));
      OD_TRY(od::launch_ns_poly(a, h->parts, it.a, it.b, it.c, std::ldexp(1.f, it.exp_s), std::ldexp(1.f, it.exp_p), st));
      if (k + 1 < steps) {
        OD_TRY(od::launch_ns_apply(a, h->parts, src, std::ldexp(1.f, it.exp_out - it.exp_p - it.exp_y), st));
      } else {
        OD_TRY(od::launch_ns_final(a, t, h->parts, src, std::ldexp(1.f, -it.exp_p - it.exp_y), update, keep, h->cfg.lr, xbf, st));
      }
    }
  }
  return ORTHDION_OK;
}

extern "C" int orthdion_muon_create(orthdion_muon_handle* out, const orthdion_muon_matdesc* mats, int32_t nmat,
                                    const orthdion_muon_config* cfg) {
  if (!out) return ORTHDION_E_NULL_PTR;
  *out = nullptr;
  orthdion_muon_handle h = nullptr;
  const int rc = no_throw([&] { return muon_create(&h, mats, nmat, cfg); });
  if (rc != ORTHDION_OK) {
    delete h;
    return rc;
  }
  *out = h;
  return ORTHDION_OK;
}

extern "C" size_t orthdion_muon_workspace_bytes(orthdion_muon_handle h) { return h ? h->ws_bytes : 0; }

extern "C" int orthdion_muon_set_lr(orthdion_muon_handle h, float lr) {
  if (!h) return ORTHDION_E_NULL_PTR;
  if (!std::isfinite(lr)) return ORTHDION_E_INVALID_ARG;
  h->cfg.lr = lr;
  return ORTHDION_OK;
}

extern "C" int orthdion_muon_set_mu(orthdion_muon_handle h, float mu) {
  if (!h) return ORTHDION_E_NULL_PTR;
  if (!std::isfinite(mu) || mu < 0.f || mu > 1.f) return ORTHDION_E_INVALID_ARG;
  h->cfg.mu = mu;
  return ORTHDION_OK;
}

extern "C" int orthdion_muon_set_weight_decay(orthdion_muon_handle h, float weight_decay) {
  if (!h) return ORTHDION_E_NULL_PTR;
  if (!std::isfinite(weight_decay)) return ORTHDION_E_INVALID_ARG;
  h->cfg.weight_decay = weight_decay;
  return ORTHDION_OK;
}

extern "C" int orthdion_muon_step(orthdion_muon_handle h, void* const* X, const void* const* G, float* const* M, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  return muon_run(h, X, G, M, true, workspace, workspace_bytes, stream);
}

extern "C" int orthdion_muon_orthogonalise(orthdion_muon_handle h, const void* const* A, void* const* O, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  return muon_run(h, O, A, nullptr, false, workspace, workspace_bytes, stream);
}

extern "C" int orthdion_muon_get_info(orthdion_muon_handle h, int32_t* info_host, void* stream) {
  if (!h || !info_host) return ORTHDION_E_NULL_PTR;
  if (!h->last_ws) return ORTHDION_E_NO_STEP;
  const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const int nmat = (int)h->mats.size();
  std::vector<int> raw;
  const int rc = no_throw([&] { raw.resize(nmat); return (int)ORTHDION_OK; });
  if (rc != ORTHDION_OK) return rc;
  OD_TRY(hipMemcpyAsync(raw.data(), reinterpret_cast<const char*>(h->last_ws) + h->off_info, raw.size() * sizeof(int), hipMemcpyDeviceToHost, st));
  OD_TRY(hipStreamSynchronize(st));
  for (int r = 0; r < nmat; ++r) info_host[h->order[r]] = raw[r];
  return ORTHDION_OK;
}

extern "C" int orthdion_muon_destroy(orthdion_muon_handle h) {
  if (!h) return ORTHDION_E_NULL_PTR;
  delete h;
  return ORTHDION_OK;
}
