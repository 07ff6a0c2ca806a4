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
using od::NsJob;

constexpr size_t kAlign = 256;
constexpr int64_t kMaxDim = 1 << 22;       // 32-bit offsets of the operand loads: 256 rows of 2^22 fp16 words
// Matrices step together (a cluster: every kernel of the iteration is one launch over it) up to this many elements; the
// next cluster reuses the workspace (24 decoder layers: 2^28 42.0, 2^29 41.0, 2^30 40.8 ms and twice the workspace).
constexpr int64_t kClusterElements = (int64_t)1 << 29;
// A slice is counted as the elements that it would be at this many words each, if those are more: thin matrices take more by the
// padding of their rows and by their partial sums (4 x 100000: 35 words an element), those of more than 128 rows up to 7.5.  So no
// cluster takes more workspace than 8.6 GB, 17.2 in two words, unless one matrix does.
constexpr int64_t kSliceWords = 8;
// Elements behind one partial sum of squares, while those are fewer than kMuonParts.  With 16384 the odd matrix of six small
// ones (201 x 327) took 24 us, the time of a thread's chain of single loads.
constexpr int64_t kPartElements = 2048;

size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
int up64(int64_t v) { return (int)((v + 63) / 64 * 64); }
// rows a multiple of 2 KB apart would put the rows of a tile on few memory channels
int pitch(int64_t v) { return up64(v) % 1024 == 0 ? up64(v) + 64 : up64(v); }

constexpr int kMostSymmetric = 5;          // symmetric matrices of a slice

// Operands of a job, in the order in which they lie in a slice: Y buffer 0 or 1, symmetric matrix 0 .., partial sums.
enum Where { IN_Y, IN_SYMMETRIC, IN_PARTIALS };
struct Operand { Where where; int index; };
struct PlannedJob {
  od::NsKind kind;
  Operand a, b, e, out;
  float ca, cb, cc;
};
// What a class does from its scaled input on: stage s of every class is one launch, the last job the final product.
struct Plan {
  std::vector<std::vector<PlannedJob>> stages;
  std::vector<od::NsSteps> steps;          // of the stages that are NS_SMALL, in order
  PlannedJob last;
  int symmetric;                           // matrices that the jobs use
};
// How: step by step, several steps on one Gram matrix, or those with all p x p work in one workgroup.
enum Mode { STEP_BY_STEP, SEGMENTS, SMALL };
constexpr int kModes = 3;

struct Class {
  NsJob job;                               // shape, slices and tables; base from the call
  size_t offset;                           // bytes of its slices behind the cluster's start
  const Plan* plan[2];                     // of the orthogonalisation and of the step
  int symmetric;                           // matrices in a slice
  int splits;                              // of its Gram matrices, 0: one sum
};
struct Cluster {
  std::vector<Class> classes;
  int mat0, count;                         // rows of the matrix tables
};

// Steps of one segment share their S = Y Y^T (see od_muon.hip).  Every S = P S P multiplies the rounding errors of S in
// the directions of small singular values by up to max |P|^2, as it multiplies those singular values themselves; what counts is
// how far that has gone where P stops being flat, a later segment starts there.  So a segment ends where the product of its
// max |P|^2 would pass a limit.  Emulated on matrices of power-law, spiked and flat spectra, relative error of O for the published
// coefficients:
//   one fp16 word, 512 x 1024 to 1528 x 3304: step by step 0.9 to 3.0e-3, cut 2 + 2 + 1 1.2 to 2.4e-3, 3 + 2 0.9 to 2.7e-3,
//   2 + 3 up to 9e-3, in one segment up to 0.5; measured on 136 x 4096 to 500 x 2000, flat, spiked, 1 / n and 1 / n^2 spectra: step by
//   step 1.1 to 3.8e-3 (1 / n^2 2.0e-2), 2 + 2 + 1 1.1 to 3.3e-3 (1.9e-2), 3 + 2 1.5 to 4.3e-3 (2.0e-2)
//   two words, 40 x 200 to 512 x 2048: step by step 1.1 to 6.1e-6, 2 + 1 + 2 1.1 to 5.2e-6, 2 + 2 + 1 1.2 to 5.2e-6 (twice as
//   much as step by step on some), 3 + 2 1.1 to 7e-6
//   one word for Y, two for the p x p work (small matrices), 40 x 200 to 300 x 700: 3 + 2 0.5 to 1.4e-3, in one segment 0.3 to 5.4e-3
constexpr double kGrowth = 13.0, kLongGrowth = 160.0;
// The long first segment (3 + 2) is taken where O does not leave with the precision of one word: by the step of a bf16 X in
// fast precision, whose 8 bits take lr O (24 decoder layers: 40.8 -> 35.6 ms; `coarse`), and by small matrices.
bool long_first(Mode mode, int parts, bool coarse) { return parts == 1 && (mode == SMALL || coarse); }
// In units of p^3 a step by itself costs 3 rho + 1 with rho = q / p, a segment of L steps 3 rho + 4 L - 3: the same for two
// segments of 3 + 2 and five steps at rho = 1.  But a segment has more and smaller launches, so matrices of few rows need long
// ones (us a step, step by step / in segments): bf16 136 x 1024 112 / 104, 136 x 16384 158 / 125, 16 of 256 x 1024 157 / 134, of 256 x 768
// 113 / 119, of 384 x 1152 209 / 193, 8 of 480 x 1440 213 / 193, of 480 x 960 154 / 168; fp32 16 of 256 x 1024 217 / 192.
constexpr int kSegmentRows = 512, kSegmentColumns = 1024;
Mode mode_for(int p, int q) {
  if (p <= od::kNsSmall) return SMALL;
  const bool segments = p >= kSegmentRows ? 4 * (int64_t)q >= 5 * (int64_t)p : q >= kSegmentColumns && q >= 3 * (int64_t)p;
  return segments ? SEGMENTS : STEP_BY_STEP;
}

// In fast precision the orthogonalisation takes two words where that costs next to nothing, in sets so small that launches
// take longer than their products (sum of p^2 q up to this): O then leaves with the error of its own rounding alone.  With one
// word O of 400 x 600 is 1.95e-3 off before bf16's 1.7e-3.  The step, whose X takes lr O, keeps one.
constexpr int64_t kTwoWordWork = (int64_t)1 << 29;

int64_t gram_tiles(int p, int64_t nb) {
  const int64_t n = (p + od::kNsSplitTile - 1) / od::kNsSplitTile;
  return n * (n + 1) / 2 * nb;
}

// Splits of the K range of a class's Gram matrices, 0: one sum.  For the kernel that adds them up by itself (SMALL), unless it
// computes them as well: its workgroup reads 64 KB a split, about as long as two steps take, so the square root of the steps
// balances the two.  Otherwise where the tiles leave most of the chip idle and the range is long: at most one round of workgroups,
// and as many splits as balance a workgroup's steps with the adding up, whose time grows with the splits and with the tiles of the
// set (`beside`).  Against eight steps a split (us, orthogonalisation, fp32): 200 x 4096 152 -> 144, 150 x 1024 139 -> 124, 4 of 200 x 1500
// 166 -> 156, 130 x 60000 316 -> 275, 4 of 512 x 4096 337 -> 301, 20 of 136 x 4096 334 -> 296, 480 x 9000 246 -> 248.
int splits_for(Mode mode, int p, int q, int nb, int64_t beside, int parts) {
  const int64_t steps = up64(q) / od::kNsStep;
  if (mode == SMALL && od::ns_small_whole(p, q, parts)) return 0;
  if (mode == SMALL) return (int)std::min<int64_t>(64, std::max<int64_t>(1, (int64_t)std::lround(std::sqrt(0.6 * (double)steps))));
  const int64_t tiles = gram_tiles(p, nb);
  if (tiles >= 128 || steps < 16) return 0;
  const int64_t depth = std::max(1L, std::lround(std::sqrt((double)steps * (double)(16 + beside) / 80.0)));       // steps of a split
  const int64_t splits = std::min<int64_t>(256 / tiles, (steps + depth - 1) / depth);
  return splits > 1 ? (int)splits : 0;
}

// power of two that brings values up to `bound` to 2^13 at most, three bits below the end of fp16's range
int exponent_for(double bound) { return 13 - (int)std::ceil(std::log2(bound)); }

}  // namespace

struct orthdion_muon_ctx {
  std::vector<orthdion_muon_matdesc> mats;
  orthdion_muon_config cfg;
  int parts[2];                            // words of a value: of the orthogonalisation, of the step
  Plan plans[2][2][kModes];                // [step][Gram matrices in partial sums][mode]
  int first_exp;                           // power of two of the scaled input
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

struct Step {
  double a, b, c;
  double top;                              // bound of the singular values it starts from
  double poly;                             // of |a + b s^2 + c s^4| over them
};

// Powers of two of the stored words follow from bounds on the spectral norms, which bound every entry: sigma <= 1 at the start
// (Frobenius norm 1), then the largest |sigma (a + b sigma^2 + c sigma^4)| over the range before, with 2 % for rounding.
// Bounds of 2^-24 and above keep every scale and every quotient of scales within fp32 (the least, of the product S S:
// 2^(5 - 2 (13 + 48)) = 2^-117), so steps that shrink X or P further are refused; a polynomial that is zero gives zeros under any scale.
constexpr double kLeastBound = 1.0 / (1 << 24);
static int plan_steps(const orthdion_muon_config& cfg, std::vector<Step>* steps) {
  double top = 1.02;
  for (int k = 0; k < cfg.steps; ++k) {
    Step s{cfg.coeffs[3 * k], cfg.coeffs[3 * k + 1], cfg.coeffs[3 * k + 2], top, 0.0};
    if (!std::isfinite(s.a) || !std::isfinite(s.b) || !std::isfinite(s.c)) return ORTHDION_E_INVALID_ARG;
    double next = 0.0;
    for (int i = 0; i <= 4096; ++i) {
      const double x = top * i / 4096, v = std::fabs(s.a + s.b * x * x + s.c * x * x * x * x);
      s.poly = std::max(s.poly, v);
      next = std::max(next, v * x);
    }
    if (!(s.poly <= 256.0) || !(next <= 32.0)) return ORTHDION_E_INVALID_ARG;
    // what the last step leaves is stored as fp32 or bf16
    if ((s.poly > 0.0 && s.poly < kLeastBound) || (k + 1 < cfg.steps && next > 0.0 && next < kLeastBound)) return ORTHDION_E_INVALID_ARG;
    s.poly = std::max(1.02 * s.poly, kLeastBound);
    top = std::max(1.02 * next, kLeastBound);
    steps->push_back(s);
  }
  steps->push_back(Step{0.0, 0.0, 0.0, top, 1.0});            // the bound behind the last step
  return ORTHDION_OK;
}

// bound of |P_0 P_1 .. P_(count - 1)| of the steps from `from` on
static double product_bound(const std::vector<Step>& steps, int from, int count) {
  double most = 0.0;
  for (int i = 0; i <= 4096; ++i) {
    double x = steps[from].top * i / 4096, z = 1.0;
    for (int k = from; k < from + count; ++k) {
      const double v = steps[k].a + steps[k].b * x * x + steps[k].c * x * x * x * x;
      z *= v;
      x *= std::fabs(v);
    }
    most = std::max(most, std::fabs(z));
  }
  return std::max(1.02 * most, kLeastBound * kLeastBound);
}

static void plan_jobs(const std::vector<Step>& steps, Mode mode, bool split, int parts, bool coarse, Plan* plan) {
  const int count = (int)steps.size() - 1;
  const Operand none{IN_SYMMETRIC, 0}, s_mat{IN_SYMMETRIC, 0}, t_mat{IN_SYMMETRIC, 1}, partials{IN_PARTIALS, 0};
  auto two = [](int e) { return (float)std::ldexp(1.0, e); };
  int src = 0;
  plan->symmetric = mode == SMALL ? 1 : 2;
  for (int k = 0; k < count;) {
    int length = 1;
    // two words: only the first and the last segment hold more than one step
    if (mode != STEP_BY_STEP && (parts == 1 || k == 0 || k + 2 == count)) {
      const double limit = k == 0 && long_first(mode, parts, coarse) ? kLongGrowth : kGrowth;
      double growth = 1.0;
      while (k + length < count) {
        growth *= steps[k + length - 1].poly * steps[k + length - 1].poly;
        if (growth > limit) break;
        ++length;
      }
    }
    const int exp_y = exponent_for(steps[k].top);
    auto apply_of = [&](const Operand& z, int exp_z) {
      const int exp_out = k + length < count ? exponent_for(steps[k + length].top) : 0;
      const PlannedJob apply{od::NS_APPLY, z, {IN_Y, src}, none, {IN_Y, 1 - src}, 0.f, 0.f, two(exp_out - exp_z - exp_y)};
      if (k + length < count) plan->stages.push_back({apply});
      else plan->last = apply;
      src = 1 - src;
      k += length;
    };
    if (mode == SMALL) {
      od::NsSteps list = {};
      list.count = length;
      for (int l = 0; l < length; ++l) {
        const Step& st = steps[k + l];
        list.a[l] = (float)st.a; list.b[l] = (float)st.b; list.c[l] = (float)st.c;
        list.s[l] = two(exponent_for(st.top * st.top));
        list.p[l] = two(exponent_for(st.poly));
        list.t[l] = two(exponent_for(st.poly * st.top * st.top));
        list.z[l] = two(exponent_for(product_bound(steps, k, l + 1)));
      }
      const Operand y{IN_Y, src};
      plan->stages.push_back({});          // the same number of stages with and without
      if (split) plan->stages.back().push_back(PlannedJob{od::NS_GRAM, y, y, none, partials, 0.f, 0.f, 1.f});
      plan->stages.push_back({PlannedJob{od::NS_SMALL, split ? partials : y, none, none, s_mat, 0.f, 0.f, two(-2 * exp_y)}});
      plan->steps.push_back(list);
      apply_of(s_mat, exponent_for(product_bound(steps, k, length)));
      continue;
    }
    // P and Z change between the matrices behind S and T (step by step: P alone, where T would be)
    Operand p_mat = length > 1 ? Operand{IN_SYMMETRIC, 2} : t_mat, z_mat = p_mat;
    if (length > 1) plan->symmetric = kMostSymmetric;
    int exp_s = exponent_for(steps[k].top * steps[k].top), exp_p = exponent_for(steps[k].poly), exp_z = exp_p;
    plan->stages.push_back({PlannedJob{od::NS_GRAM, {IN_Y, src}, {IN_Y, src}, none, split ? partials : s_mat, 0.f, 0.f, two(exp_s - 2 * exp_y)}});
    if (split) plan->stages.push_back({PlannedJob{od::NS_REDUCE, partials, none, none, s_mat, 0.f, 0.f, two(exp_s - 2 * exp_y)}});
    auto poly = [&](const Step& st, Operand out) {
      return PlannedJob{od::NS_SYM, s_mat, s_mat, s_mat, out, (float)(st.a * two(exp_p)), (float)(st.b * two(exp_p - exp_s)), (float)(st.c * two(exp_p - 2 * exp_s))};
    };
    plan->stages.push_back({poly(steps[k], p_mat)});
    for (int l = 1; l < length; ++l) {
      const Step& before = steps[k + l - 1];
      const Step& st = steps[k + l];
      // T = P S; and Z = P Z of the step before, unless it is P itself
      const int exp_t = exponent_for(before.poly * before.top * before.top);
      std::vector<PlannedJob> pair{PlannedJob{od::NS_SYM, p_mat, s_mat, none, t_mat, 0.f, 0.f, two(exp_t - exp_p - exp_s)}};
      Operand new_z = z_mat;
      if (l > 1) {
        const int exp_new = exponent_for(product_bound(steps, k, l));
        new_z = Operand{IN_SYMMETRIC, 2 + 3 + 4 - p_mat.index - z_mat.index};
        pair.push_back(PlannedJob{od::NS_FULL, p_mat, z_mat, none, new_z, 0.f, 0.f, two(exp_new - exp_p - exp_z)});
        exp_z = exp_new;
      }
      plan->stages.push_back(pair);
      // S = T P
      const int exp_new_s = exponent_for(st.top * st.top);
      plan->stages.push_back({PlannedJob{od::NS_SYM, t_mat, p_mat, none, s_mat, 0.f, 0.f, two(exp_new_s - exp_t - exp_p)}});
      exp_s = exp_new_s;
      // the next P where neither Z nor, for its last use, the old P lies
      z_mat = new_z;
      exp_p = exponent_for(st.poly);
      int index = 2;
      while (index == z_mat.index) ++index;
      p_mat = Operand{IN_SYMMETRIC, index};
      plan->stages.push_back({poly(st, p_mat)});
    }
    if (length > 1) {
      const int exp_new = exponent_for(product_bound(steps, k, length));
      const Operand new_z{IN_SYMMETRIC, 2 + 3 + 4 - p_mat.index - z_mat.index};
      // not mirrored: the two orders of the rounded factors differ by their commutator, and one triangle of each would
      // leave more than either (1528 x 3304, cut 2 + 2 + 1: 1.54e-3 mirrored, 1.34e-3 not)
      plan->stages.push_back({PlannedJob{od::NS_FULL, p_mat, z_mat, none, new_z, 0.f, 0.f, two(exp_new - exp_p - exp_z)}});
      z_mat = new_z;
      exp_z = exp_new;
    }
    apply_of(z_mat, exp_z);
  }
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
  std::vector<Step> steps;
  if ((rc = plan_steps(*cfg, &steps)) != ORTHDION_OK) return rc;
  h->first_exp = exponent_for(steps[0].top);
  const bool exact = cfg->precision == ORTHDION_PREC_EXACT ||
                     (cfg->precision == ORTHDION_PREC_AUTO && !(cfg->x_dtype == ORTHDION_BF16 && cfg->g_dtype == ORTHDION_BF16));
  // classes in order of first appearance
  struct Shape { int p, q, tall; std::vector<int> members; };
  std::vector<Shape> classes;
  for (int i = 0; i < nmat; ++i) {
    const int p = (int)std::min(mats[i].m, mats[i].n), q = (int)std::max(mats[i].m, mats[i].n), tall = mats[i].m > mats[i].n;
    size_t k = 0;
    while (k < classes.size() && !(classes[k].p == p && classes[k].q == q && classes[k].tall == tall)) ++k;
    if (k == classes.size()) classes.push_back(Shape{p, q, tall, {}});
    classes[k].members.push_back(i);
  }
  bool all_small = true;
  // Beside larger matrices small ones ride along in their launches, which are there anyway: six matrices of 128 to 392 rows
  // 209 us a step, with launches of their own kernel in between 275.
  auto mode_of = [&](const Shape& c) {
    const Mode mode = mode_for(c.p, c.q);
    return mode == SMALL && !all_small ? STEP_BY_STEP : mode;
  };
  for (const Shape& c : classes) all_small = all_small && mode_for(c.p, c.q) == SMALL;
  double work = 0.0;
  for (const Shape& c : classes) work += (double)c.p * c.p * c.q * (double)c.members.size();
  h->parts[0] = exact || (!all_small && work <= (double)kTwoWordWork) ? 2 : 1;
  h->parts[1] = exact ? 2 : 1;
  const bool coarse[2] = {false, cfg->x_dtype == ORTHDION_BF16};
  for (int step = 0; step < 2; ++step)
    for (int split = 0; split < 2; ++split)
      for (int mode = 0; mode < kModes; ++mode) plan_jobs(steps, (Mode)mode, split != 0, h->parts[step], coarse[step], &h->plans[step][split][mode]);
  // Splits; where those of the set would take more than two workgroups a CU, fewer of each (a 1024-wide model in fp32, 576 workgroups
  // 791 us a step, 432 688)
  int64_t beside = 0, groups = 0;
  for (const Shape& c : classes) beside += gram_tiles(c.p, (int64_t)c.members.size());
  std::vector<int> splits_of;
  for (const Shape& c : classes) {
    splits_of.push_back(splits_for(mode_of(c), c.p, c.q, (int)c.members.size(), beside, h->parts[0]));
    groups += gram_tiles(c.p, (int64_t)c.members.size()) * splits_of.back();
  }
  if (!all_small && groups > 512)
    for (int& splits : splits_of) splits = (int)(splits * (int64_t)512 / groups) > 1 ? (int)(splits * (int64_t)512 / groups) : 0;
  // clusters
  int64_t held = 0;
  size_t slices = 0, most = 0;
  for (const Shape& c : classes) {
    const int lp = pitch(c.p), lq = pitch(c.q);
    const Mode mode = mode_of(c);
    // O in one word of few rows, leaving with that precision: 2 + 2 + 1 steps left 2.6 to 3.4e-3 on 136 x 16384 of a falling spectrum, step by step 2.2e-3 (bf16's rounding
    // alone 1.7e-3)
    auto mode_of_call = [&](int step) { return mode == SEGMENTS && c.p < kSegmentRows && h->parts[step] == 1 && !coarse[step] ? STEP_BY_STEP : mode; };
    const int splits = splits_of[&c - classes.data()];
    const Plan* const plan[2] = {&h->plans[0][splits > 0][mode_of_call(0)], &h->plans[1][splits > 0][mode_of_call(1)]};
    const int symmetric = std::max(plan[0]->symmetric, plan[1]->symmetric);
    const int64_t stride = h->parts[0] * (2 * od::ns_y_plane(c.p, lq) + symmetric * od::ns_s_plane(c.p, lp)) + od::ns_partials(c.p, splits);
    const int64_t elements = std::max((int64_t)c.p * c.q, stride / (kSliceWords * h->parts[0]));
    for (size_t done = 0; done < c.members.size();) {
      if (h->clusters.empty() || held + elements > kClusterElements || (int)h->clusters.back().classes.size() == od::kNsClasses) {
        h->clusters.push_back(Cluster{});
        h->clusters.back().mat0 = (int)h->order.size();
        held = 0;
        slices = 0;
      }
      Cluster& cl = h->clusters.back();
      const int64_t room = std::max((int64_t)1, (kClusterElements - held) / elements);
      // the workgroups of a launch are counted in 32 bits: a class of many matrices is 64 x 64 tiles at least
      const int take = (int)std::min<int64_t>({room, (int64_t)(c.members.size() - done), 1 << 20});
      NsJob job = {};
      job.p = c.p; job.q = c.q; job.lp = lp; job.lq = lq; job.nb = take; job.tall = c.tall;
      job.mat0 = (int)h->order.size();
      job.stride = stride;
      cl.classes.push_back(Class{job, slices, {plan[0], plan[1]}, symmetric, splits});
      slices = align_up(slices + (size_t)take * (size_t)stride * 2);
      most = std::max(most, slices);
      for (int k = 0; k < take; ++k) {
        const int i = c.members[done + k];
        const orthdion_muon_matdesc& d = mats[i];
        // rows are dealt out first; a matrix of few rows is cut across its columns too, in ranges of a multiple of 8
        const int64_t want = std::min<int64_t>((d.m * d.n + kPartElements - 1) / kPartElements, od::kMuonParts);
        const int64_t rows = std::min<int64_t>(want, d.m), cols = std::min<int64_t>(want / rows, (d.n + 7) / 8);
        h->order.push_back(i);
        h->table.push_back(MuonMat{(int)d.m, (int)d.n, d.ldx, d.ldg, d.ldm, d.scale, (int)(rows * cols), (int)cols});
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

// The launches of one cluster behind the input's norm, in order: f(what, jobs, steps of a NS_SMALL launch).
enum Launch { SCALE, PRODUCTS, REDUCE, SMALL_STEPS, LAST };
template <class F>
static int for_launches(orthdion_muon_handle h, const Cluster& cl, bool update, char* slices, F&& f) {
  const int parts = h->parts[update];
  NsArgs args;
  auto add = [&](const Class& c, const PlannedJob& job) {
    NsJob& j = args.j[args.count++];
    j = c.job;
    j.base = reinterpret_cast<uint16_t*>(slices + c.offset);
    auto at = [&](const Operand& o) {
      const int64_t y = od::ns_y_plane(j.p, j.lq) * parts, s = od::ns_s_plane(j.p, j.lp) * parts;
      return o.where == IN_Y ? o.index * y : 2 * y + (o.where == IN_SYMMETRIC ? o.index : c.symmetric) * s;
    };
    j.kind = job.kind;
    j.a = at(job.a); j.b = at(job.b); j.e = at(job.e); j.out = at(job.out);
    j.ca = job.ca; j.cb = job.cb; j.cc = job.cc;
    j.splits = job.kind == od::NS_GRAM || job.kind == od::NS_REDUCE || job.kind == od::NS_SMALL ? c.splits : 0;
  };
  args.count = 0;
  size_t stages = 0;
  for (const Class& c : cl.classes) {
    add(c, c.plan[update]->last);
    stages = std::max(stages, c.plan[update]->stages.size());
  }
  OD_TRY(f(SCALE, args, nullptr));
  const NsArgs last = args;
  // the jobs of stage s that `of` takes; the plan of the last of them
  auto gather = [&](size_t s, auto&& of) {
    const Plan* plan = nullptr;
    args.count = 0;
    for (const Class& c : cl.classes)
      if (s < c.plan[update]->stages.size())
        for (const PlannedJob& job : c.plan[update]->stages[s])
          if (of(job.kind)) {
            add(c, job);
            plan = c.plan[update];
          }
    return plan;
  };
  for (size_t s = 0; s < stages; ++s) {
    if (gather(s, [](od::NsKind k) { return k <= od::NS_FULL; })) OD_TRY(f(PRODUCTS, args, nullptr));
    if (gather(s, [](od::NsKind k) { return k == od::NS_REDUCE; })) OD_TRY(f(REDUCE, args, nullptr));
    // small matrices take three stages a segment
    if (const Plan* plan = gather(s, [](od::NsKind k) { return k == od::NS_SMALL; })) OD_TRY(f(SMALL_STEPS, args, &plan->steps[s / 3]));
  }
  OD_TRY(f(LAST, last, nullptr));
  return ORTHDION_OK;
}

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
  const int parts = h->parts[update];
  for (const Cluster& cl : h->clusters) {
    OD_TRY(od::launch_muon_begin(entries.get() + cl.mat0, h->table.data() + cl.mat0, cl.mat0, cl.count, t, h->cfg.mu, nesterov, gbf, st));
    const int rc = for_launches(h, cl, update, ws + h->off_slices, [&](Launch what, const NsArgs& args, const od::NsSteps* steps) {
      switch (what) {
        case SCALE: return od::launch_muon_scale(args, t, h->cfg.mu, nesterov, gbf, parts, h->cfg.eps, std::ldexp(1.0, h->first_exp), st);
        case PRODUCTS: return od::launch_ns_products(args, parts, st);
        case REDUCE: return od::launch_ns_reduce(args, parts, st);
        case SMALL_STEPS: return od::launch_ns_small(args, *steps, parts, st);
        default: return od::launch_ns_final(args, t, parts, update, keep, h->cfg.lr, xbf, st);
      }
    });
    if (rc != ORTHDION_OK) return rc;
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

extern "C" int orthdion_muon_get_tiles(orthdion_muon_handle h, int32_t step, int32_t* tiles) {
  if (!h || !tiles) return ORTHDION_E_NULL_PTR;
  if (step != 0 && step != 1) return ORTHDION_E_INVALID_ARG;
  for (int k = 0; k < ORTHDION_MUON_PRODUCTS; ++k) tiles[k] = 0;
  for (const Cluster& cl : h->clusters) {
    const int rc = for_launches(h, cl, step != 0, nullptr, [&](Launch what, const NsArgs& args, const od::NsSteps*) {
      if (what == PRODUCTS || what == LAST) {
        const int bit = 1 << (od::ns_tile(args, h->parts[step]) / 64 - 1);
        for (int k = 0; k < args.count; ++k) tiles[what == PRODUCTS ? args.j[k].kind : args.j[k].tall ? 5 : 4] |= bit;
      }
      return hipSuccess;
    });
    if (rc != ORTHDION_OK) return rc;
  }
  return ORTHDION_OK;
}

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
