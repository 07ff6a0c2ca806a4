// Launchers of the Muon kernels (od_muon.hip): momentum and scaling of the input, the products of the
// Newton-Schulz iteration, the parameter update.  Every launcher only enqueues work on `stream`.
//
// A matrix A (m x n) is worked on as Y (p x q) with p = min(m, n), q = max(m, n): A itself or its transpose.
// Its slice of the workspace holds fp16 operand words only, `parts` planes (1: the value under a power-of-two
// scale, 2: hi + lo of it) of
//   Y twice (read by one product, written by another)   pp rows of lq, rows p .. pp and columns q .. qq zero
//   symmetric p x p matrices                             p rows of lp, columns p .. pp zero
// with pp and qq the multiples of 64 above p and q: the K loops run over whole 64-deep steps unchecked.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace od {

constexpr int kNsStep = 64;                // k of one step of the K loops
constexpr int kNsClasses = 16;             // classes (matrices of one shape) that step together
constexpr int kNsJobs = 2 * kNsClasses;    // jobs of one launch: up to two per class
constexpr int kMuonChunk = 48;             // matrices whose pointers travel in one launch's arguments
constexpr int kMuonParts = 256;            // most partial sums of squares of one matrix

// caller's buffers of one matrix; O and A of orthdion_muon_orthogonalise stand at X and G, M is null
struct MuonEntry {
  void* X;
  const void* G;
  float* M;
};

struct MuonMat {                           // one matrix, as the elementwise kernels see it
  int m, n;
  int64_t ldx, ldg, ldm;
  float scale;                             // of its update
  int blocks;                              // partial sums: row ranges times column ranges
  int col_ranges;
};

// What a launch computes for one class: nb matrices of p x q (or q x p where tall).
enum NsKind : int {
  NS_GRAM = 0,                             // out = cc a a^T of Y at a
  NS_SYM = 1,                              // out = ca I + cb e + cc a b of commuting symmetric a, b; e read where cb != 0
  NS_APPLY = 2,                            // out = cc a b of p x p a and Y at b
  NS_FULL = 3,                             // out = cc a b of symmetric a, b, not mirrored
  NS_REDUCE = 4,                           // out = cc (sum of the partial sums at a)
  NS_SMALL = 5                             // out = Z of a segment of steps from cc (sum of the partial sums at a; splits 0: a a^T of Y at a)
};
struct NsJob {
  int first;                               // first workgroup of the job
  int p, q, lp, lq, nb;
  int mat0;                                // first row of the class in the matrix tables
  int tall;
  uint16_t* base;                          // slice of the class's first matrix
  int64_t stride;                          // elements between slices
  int64_t a, b, e, out;                    // operands in a slice, elements
  float ca, cb, cc;
  int kind;
  int splits;                              // NS_GRAM: > 0: that many partial sums of the K range, fp32 at out, for another
                                           // kernel to add up
};

template <int N>
struct NsJobs {
  int count, total;                        // jobs, workgroups
  NsJob j[N];
};
typedef NsJobs<kNsJobs> NsArgs;            // with the tables' pointers below the 4 KB of a launch's arguments

// elements of a slice
inline int64_t ns_y_plane(int p, int lq) { return (int64_t)((p + kNsStep - 1) / kNsStep * kNsStep) * lq; }
inline int64_t ns_s_plane(int p, int lp) { return (int64_t)p * lp; }

// Partial sums of a matrix: [tile of the upper triangle][split][kNsSplitTile * kNsSplitTile], row by row, rounded up to whole
// groups of kNsStep fp16 words.
constexpr int kNsSplitTile = 128;
inline int64_t ns_partials(int p, int splits) {
  const int64_t n = (p + kNsSplitTile - 1) / kNsSplitTile;
  return n * (n + 1) / 2 * splits * kNsSplitTile * kNsSplitTile * 2;
}

// Steps of a segment for the kernel that does all p x p work of a small matrix in LDS: coefficients and the powers of two
// of the words of S, P, T = P S and Z that step k writes.
constexpr int kNsSmall = 128;              // largest p
inline int ns_small_size(int p) { return (p + 31) / 32 * 32; }
// Whether that kernel computes the Gram matrix as well: Y then fits where the words of S and P will lie, 16 bytes a row for the
// LDS banks included.  96 x 160 in two words: 82.4 us a call with launches of their own for the Gram matrices, 69.2 so.
inline bool ns_small_whole(int p, int q, int parts) { return parts * ((q + kNsStep - 1) / kNsStep * kNsStep) <= 4 * ns_small_size(p); }
constexpr int kNsMostSteps = 32;
struct NsSteps {
  int count;
  float a[kNsMostSteps], b[kNsMostSteps], c[kNsMostSteps], s[kNsMostSteps], p[kNsMostSteps], t[kNsMostSteps], z[kNsMostSteps];
};

struct MuonTables {                        // in the workspace, one row per matrix
  MuonEntry* entries;
  const MuonMat* mats;
  double* partials;                        // kMuonParts per matrix
  int* info;                               // 1: a non-finite entry
};

// width of the tiles that the products of a launch are computed on
int ns_tile(const NsArgs& a, int parts);

// M = mu M + G and the partial sums of squares of B; copies the pointers and shapes of `count` matrices
// (rows mat0 ..) into the tables.  entries[i].M null: B = G.
hipError_t launch_muon_begin(const MuonEntry* entries, const MuonMat* mats, int mat0, int count, const MuonTables& t, float mu,
                             bool nesterov, bool g_bf16, hipStream_t st);
// Y = B * (scale / (||B||_F + eps)) in fp16 words, zero padding, info words; one job per class
hipError_t launch_muon_scale(const NsArgs& a, const MuonTables& t, float mu, bool nesterov, bool g_bf16, int parts, double eps,
                             double scale, hipStream_t st);
// jobs of kinds up to NS_FULL; of NS_REDUCE; of NS_SMALL (one list of steps for all)
hipError_t launch_ns_products(const NsArgs& a, int parts, hipStream_t st);
hipError_t launch_ns_reduce(const NsArgs& a, int parts, hipStream_t st);
// p up to kNsSmall
hipError_t launch_ns_small(const NsArgs& a, const NsSteps& steps, int parts, hipStream_t st);
// O = cc a b of jobs of kind NS_APPLY, into the callers' matrices: X = O, or with `update` X = keep X - lr scale_i O
hipError_t launch_ns_final(const NsArgs& a, const MuonTables& t, int parts, bool update, float keep, float lr, bool x_bf16, hipStream_t st);

}  // namespace od
