// Muon: Newton-Schulz orthogonalisation of a set of matrices and the optimizer step around it (the method's
// published form: quintic iteration on the Frobenius-normalised momentum).  For every matrix
//   M  = mu M + G,   B = G + mu M (Nesterov) or M
//   X0 = B / (||B||_F + eps)
//   S  = Xk Xk^T,   P = a I + b S + c S S,   Xk+1 = P Xk        K times
//   X  = (1 - lr wd) X - lr scale XK
// S, S S and P are symmetric: only tiles on and above the diagonal are computed, the others mirrored.  All polynomials in
// S commute, so several steps can share one S = Xk Xk^T and one product with Xk:
//   Z = P,  then per further step  S = P S P,  P = a I + b S + c S S,  Z = P Z,  and at last  Xk+L = Z Xk
// (which steps do is the host's plan).  See od_muon.h for the layout of the workspace.
#include "od_muon.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "od_dma.h"

namespace od {

typedef short s16x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------------------------
// Elementwise kernels
// ------------------------------------------------------------------------------------
template <bool BF>
OD_DEV float load_elem(const void* p, int64_t i) {
  if constexpr (BF) return bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(p)[i]);
  else return reinterpret_cast<const float*>(p)[i];
}

// eight consecutive elements, 16-byte aligned
template <bool BF>
OD_DEV void load8(const void* p, int64_t i, float* x) {
  if constexpr (BF) SrcBF16::unpack8(*reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(p) + i), x);
  else {
    const f32x4* q = reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(p) + i);
    SrcF32::unpack8(SrcF32::Raw8{q[0], q[1]}, x);
  }
}

OD_DEV bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// whether eight consecutive elements of any row can be moved at once
OD_DEV bool rows_aligned(const void* p, int64_t ld) { return aligned16(p) && (ld & 7) == 0; }

struct MuonChunk {
  MuonEntry e[kMuonChunk];
  MuonMat m[kMuonChunk];
};

// sum over the workgroup's 256 threads, in every thread
OD_DEV double block_sum(double v, double* lds) {
  for (int s = 1; s < kWave; s <<= 1) v += __shfl_xor(v, s);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// One workgroup: a range of rows and columns of one matrix.  HBM bound: G read, M read and written.
template <bool GBF>
__global__ __launch_bounds__(256) void k_muon_begin(MuonChunk chunk, MuonTables t, int mat0, float mu, int nesterov) {
  __shared__ double lds[4];
  const int z = blockIdx.y;
  const MuonMat a = chunk.m[z];
  const MuonEntry e = chunk.e[z];
  if ((int)blockIdx.x >= a.blocks) return;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    t.entries[mat0 + z] = e;
    const_cast<MuonMat*>(t.mats)[mat0 + z] = a;
  }
  const int row_ranges = a.blocks / a.col_ranges, ri = blockIdx.x / a.col_ranges, ci = blockIdx.x % a.col_ranges;
  const int64_t rows = ((int64_t)a.m + row_ranges - 1) / row_ranges;
  const int64_t r0 = ri * rows, r1 = min((int64_t)a.m, r0 + rows);
  const int cols = ((a.n + 7) / 8 + a.col_ranges - 1) / a.col_ranges * 8, n0 = min(a.n, ci * cols), n1 = min(a.n, n0 + cols);
  double sum = 0.0;
  const bool vec = rows_aligned(e.G, a.ldg) && (e.M == nullptr || rows_aligned(e.M, a.ldm));
  // threads side by side along a row: the power of two at or above its items, so that narrow rows share a wave
  const int wide = vec ? (n1 - n0) / 8 : 0;                 // whole groups of eight
  auto spread = [](int items) { int s = 1; while (s < 256 && s < items) s <<= 1; return s; };
  if (wide > 0) {
    const int tx = spread(wide), x = threadIdx.x & (tx - 1), y = threadIdx.x / tx, ty = 256 / tx;
    for (int64_t r = r0 + y; r < r1; r += ty)
      for (int c = x; c < wide; c += tx) {
        float g[8];
        load8<GBF>(e.G, r * a.ldg + n0 + 8 * c, g);
        if (e.M) {
          float m[8];
          f32x4* mp = reinterpret_cast<f32x4*>(e.M + r * a.ldm + n0 + 8 * c);
          SrcF32::unpack8(SrcF32::Raw8{mp[0], mp[1]}, m);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            m[i] = mu * m[i] + g[i];
            const float b = nesterov ? g[i] + mu * m[i] : m[i];
            sum += (double)b * b;
          }
          mp[0] = f32x4{m[0], m[1], m[2], m[3]};
          mp[1] = f32x4{m[4], m[5], m[6], m[7]};
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) sum += (double)g[i] * g[i];
        }
      }
  }
  const int c0 = n0 + 8 * wide, rest = n1 - c0;
  if (rest > 0) {
    const int tx = spread(rest), x = threadIdx.x & (tx - 1), y = threadIdx.x / tx, ty = 256 / tx;
    for (int64_t r = r0 + y; r < r1; r += ty)
      for (int c = c0 + x; c < n1; c += tx) {
        const float g = load_elem<GBF>(e.G, r * a.ldg + c);
        float b = g;
        if (e.M) {
          const float m = mu * e.M[r * a.ldm + c] + g;
          e.M[r * a.ldm + c] = m;
          b = nesterov ? g + mu * m : m;
        }
        sum += (double)b * b;
      }
  }
  sum = block_sum(sum, lds);
  if (threadIdx.x == 0) t.partials[(int64_t)(mat0 + z) * kMuonParts + blockIdx.x] = sum;
}

OD_DEV uint32_t pack_f16(float lo, float hi) {
  f16x2 p;
  p[0] = (_Float16)lo;
  p[1] = (_Float16)hi;
  return __builtin_bit_cast(uint32_t, p);
}

// Value in fp16 words: hi, and with two parts the remainder.  The scales keep every value below 2^14, so nothing
// saturates; a NaN stays one.
template <int PARTS>
OD_DEV void split2(float a, float b, uint32_t* out) {
  out[0] = pack_f16(a, b);
  if constexpr (PARTS == 2) {
    const f16x2 h = __builtin_bit_cast(f16x2, out[0]);
    out[1] = pack_f16(a - (float)h[0], b - (float)h[1]);
  }
}

template <int N>
OD_DEV int ns_job(const NsJobs<N>& a, int bid) {
  int k = 0;
  while (k + 1 < a.count && bid >= a.j[k + 1].first) ++k;
  return k;
}

// Uniform integer division runs on the vector units; this brings its results back to scalar registers, where addresses
// and loop counts belong.
OD_DEV int quotient(int a, int b) { return __builtin_amdgcn_readfirstlane(a / b); }

OD_DEV int up64(int v) { return (v + 63) & ~63; }

// One workgroup: a 64 x 64 tile of Y (transposed on the way through LDS where the matrix is tall).  HBM bound.
template <bool GBF, int PARTS>
__global__ __launch_bounds__(256) void k_muon_scale(NsArgs args, MuonTables t, float mu, int nesterov, double eps, double scale) {
  __shared__ double lds[4];
  __shared__ float tile[64][65];
  const NsJob c = args.j[ns_job(args, blockIdx.x)];
  const int pp = up64(c.p), qq = up64(c.q), ti_n = pp / 64, tj_n = qq / 64;
  const int in_class = blockIdx.x - c.first, z = in_class / (ti_n * tj_n), tl = in_class % (ti_n * tj_n);
  const int ti = tl / tj_n, tj = tl % tj_n;
  const MuonMat a = t.mats[c.mat0 + z];
  const MuonEntry e = t.entries[c.mat0 + z];
  const int tid = threadIdx.x;
  double part = 0.0;
  for (int i = tid; i < a.blocks; i += 256) part += t.partials[(int64_t)(c.mat0 + z) * kMuonParts + i];
  const double norm = sqrt(block_sum(part, lds)) + eps;
  const bool bad = !(norm < INFINITY);
  if (tl == 0 && tid == 0) t.info[c.mat0 + z] = bad ? 1 : 0;
  const double inv = norm > 0.0 ? scale / norm : 0.0;

  // the tile of the matrix in its own orientation
  const int r0 = c.tall ? tj * 64 : ti * 64, c0 = c.tall ? ti * 64 : tj * 64;
  const bool vec = rows_aligned(e.G, a.ldg) && (e.M == nullptr || rows_aligned(e.M, a.ldm));
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int row = half * 32 + tid / 8, col = tid % 8 * 8;
    const int r = r0 + row, cc = c0 + col;
    float b[8];
    if (r < a.m && cc + 8 <= a.n && vec) {
      load8<GBF>(e.G, (int64_t)r * a.ldg + cc, b);
      if (e.M) {
        float m[8];
        load8<false>(e.M, (int64_t)r * a.ldm + cc, m);
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = nesterov ? b[i] + mu * m[i] : m[i];
      }
    } else {
      // single elements at clamped addresses, all in flight (behind a branch each they came one by one: 10 us for 201 x 327)
      const int64_t rr = min(r, a.m - 1);
      float m[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) b[i] = load_elem<GBF>(e.G, rr * a.ldg + min(cc + i, a.n - 1));
      if (e.M) {
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = e.M[rr * a.ldm + min(cc + i, a.n - 1)];
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = nesterov ? b[i] + mu * m[i] : m[i];
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // in 64 bits: the scale over the norm can leave the range of 32 where the entries are tiny
      const float y = bad ? NAN : (float)((double)b[i] * inv);
      const bool inside = r < a.m && cc + i < a.n;
      if (c.tall) tile[col + i][row] = inside ? y : 0.f;
      else tile[row][col + i] = inside ? y : 0.f;
    }
  }
  __syncthreads();
  const int64_t plane = (int64_t)pp * c.lq;
  uint16_t* y = c.base + z * c.stride;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int row = half * 32 + tid / 8, col = tid % 8 * 8;
    u32x4 w[PARTS];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t s[PARTS];
      split2<PARTS>(tile[row][col + 2 * i], tile[row][col + 2 * i + 1], s);
#pragma unroll
      for (int k = 0; k < PARTS; ++k) w[k][i] = s[k];
    }
    const int r = ti * 64 + row;
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      uint16_t* out = y + k * plane + (int64_t)r * c.lq + tj * 64 + col;
      *reinterpret_cast<u32x4*>(out) = w[k];
      // the rows beyond p of the second buffer, which no product writes
      if (r >= c.p) *reinterpret_cast<u32x4*>(out + PARTS * plane) = u32x4{0u, 0u, 0u, 0u};
    }
  }
}

// ------------------------------------------------------------------------------------
// The products.  One workgroup computes a T x T tile of C = A B over 64-deep steps; A has k along its rows, B is given
// either as the rows of B^T with k along them (TRB = false) or as rows of B, k down its columns (TRB = true).  Both
// operands come by direct-to-LDS loads into a ring of operand tiles (A0 B0 A1 B1 ..):
//   k along rows   128-byte rows, their 16-byte k-groups XOR-swizzled by (row >> 1) & 7: the 16 lanes that a
//                  ds_read_b128 serves at a time lie in 16 different groups of four banks
//   k down columns rows of T elements, their 64-byte blocks XOR-swizzled by k, so that the four rows of a
//                  ds_read_b64_tr_b16 lie in different banks
// ------------------------------------------------------------------------------------
// As dma16, from a uniform base plus 32-bit lane offsets; all lanes of the wave are active, and `mask` (all ones or zero)
// takes the load away without a branch, past which accumulators would be moved about.
OD_DEV void dma16_at(uint32_t voff, const void* sbase, uint32_t lds_base, uint32_t mask) {
  const uint32_t l = __builtin_amdgcn_readfirstlane(lds_base), m = __builtin_amdgcn_readfirstlane(mask);
  asm volatile("s_mov_b32 m0, %2\n\ts_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\tglobal_load_lds_dwordx4 %0, %1\n\ts_mov_b64 exec, -1\n" ::"v"(voff), "s"(sbase), "s"(l), "s"(m) : "memory");
}

// f(0), f(1), .. f(N - 1) with the index a constant, so that register arrays stay registers
template <int N, int I = 0, class F>
OD_DEV void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<N, I + 1>(f);
  }
}

OD_DEV int swz64(int row) { return (row >> 1) & 7; }
// what the 16-byte slots of row k of a tile with k down its columns are XORed with: rows of 128 or 384 bytes lie in alternate
// halves of the 256 bytes of all banks already
template <int T>
OD_DEV int swz_down(int k) { return T % 128 ? (k & 2) << 1 : (k & 3) << 2; }

struct NsOperand {
  const uint16_t* p;      // tile's first row (TRB: column)
  int64_t plane;          // elements between parts
  int ld;
  int rows;               // rows (TRB: columns) from the tile's first one that may be read, at least 1 (TRB: 8)
};

// The loads run two steps ahead (four gained nothing anywhere).
template <int T_, int WI_, int WJ_>
struct NsTile {
  static constexpr int T = T_, WI = WI_, WJ = WJ_, NW = WI * WJ, THREADS = 64 * NW;
  static constexpr int WTM = T / WI, WTN = T / WJ, FM = WTM / 32, FN = WTN / 32;
  static constexpr int OPER = T * 128, RING = 5;                              // bytes of an operand tile of one part
  static constexpr int CH = T / 8 / NW;                                       // 1 KB loads per wave and such a tile
  // Two parts of a value: both in the ring, three products from one load of each, where that fits LDS (1024 x 1024, a product
  // of S: 34 us in three passes); otherwise three passes over K, hi hi, hi lo and lo hi.
  static constexpr bool together(int parts) { return parts == 2 && T <= 128; }
  static constexpr int unit(int parts) { return together(parts) ? 2 * OPER : OPER; }
  static constexpr int lds(int parts) { return RING * unit(parts); }
  static constexpr int blocks(int parts) { return lds(parts) <= 81920 ? 2 : 1; }        // workgroups per CU
};

// ACROSS: the accumulator of lane l holds C[l % 32][4 consecutive columns], otherwise C[4 consecutive rows][l % 32]
template <class TL, int PARTS, bool TRB, bool ACROSS>
OD_DEV void ns_product(f32x16 (&acc)[TL::FM][TL::FN], const NsOperand& A, const NsOperand& B, int kdim, char* lds, int split = 0, int splits = 1) {
  constexpr bool BOTH = TL::together(PARTS);
  constexpr int T = TL::T, CH = TL::CH, UNIT = TL::unit(PARTS), LOADS = BOTH ? 2 * CH : CH;      // a wave's loads of a unit
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wi = wave / TL::WJ, wj = wave % TL::WJ;
  const uint32_t lds0 = lds_offset_of(lds);
  uint32_t va[CH], vb[CH];
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int chunk = wave * CH + j;
    const int row = chunk * 8 + (lane >> 3), kg = (lane & 7) ^ swz64(row);
    va[j] = (uint32_t)min(row, A.rows - 1) * (uint32_t)(A.ld * 2) + kg * 16;
    if constexpr (TRB) {
      constexpr int SLOTS = T / 8;                       // 16-byte groups of a row
      const int k = (chunk * 64 + lane) / SLOTS, cg = ((chunk * 64 + lane) % SLOTS) ^ swz_down<T>(k);
      vb[j] = (uint32_t)k * (uint32_t)(B.ld * 2) + min(cg * 8, B.rows - 8) * 2;
    } else {
      vb[j] = (uint32_t)min(row, B.rows - 1) * (uint32_t)(B.ld * 2) + kg * 16;
    }
  }
  const int ks = kdim / kNsStep, all = ks * (PARTS == 2 && !BOTH ? 3 : 1);
  // steps first .. of all, this split's share
  const int first = splits > 1 ? quotient(all * split, splits) : 0, steps = (splits > 1 ? quotient(all * (split + 1), splits) : all) - first;
  const int64_t bstep = TRB ? (int64_t)kNsStep * B.ld : kNsStep;
  // loads of one unit of one step; of a step past the last one, none
  struct Loads { const uint16_t *p, *lo; uint32_t at, mask; };
  auto slot = [&](int unit) { return (uint32_t)(unit % TL::RING) * UNIT; };
  auto loads_of = [&](int step, bool of_b) {
    const int seg = PARTS == 2 && !BOTH ? quotient(first + step, ks) : 0, kk = first + step - seg * ks;
    const uint16_t* p = of_b ? B.p + (seg == 1 ? B.plane : 0) + kk * bstep : A.p + (seg == 2 ? A.plane : 0) + (int64_t)kk * kNsStep;
    return Loads{p, p + (of_b ? B.plane : A.plane), lds0 + slot(2 * step + of_b) + wave * CH * 1024, step < steps ? ~0u : 0u};
  };
  auto issue = [&](const Loads& l, const uint32_t (&voff)[CH], auto jj) {
    constexpr int j = decltype(jj)::value;
    if constexpr (j < CH) dma16_at(voff[j], l.p, l.at + j * 1024, l.mask);
    else dma16_at(voff[j - CH], l.lo, l.at + TL::OPER + (j - CH) * 1024, l.mask);
  };
#pragma unroll
  for (int i = 0; i < TL::FM; ++i)
#pragma unroll
    for (int j = 0; j < TL::FN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

  constexpr int HL = BOTH ? 2 : 1;
  u32x4 fa[2][HL][TL::FM], fb[2][HL][TL::FN];
  auto fetch = [&](int step, int sub, auto ss) {
    constexpr int set = decltype(ss)::value;
    const char* at_a = lds + slot(2 * step);
    const char* at_b = lds + slot(2 * step + 1);
    const int kg = 2 * sub + (lane >> 5);
#pragma unroll
    for (int h = 0; h < HL; ++h) {
#pragma unroll
      for (int i = 0; i < TL::FM; ++i) {
        const int row = wi * TL::WTM + 32 * i + (lane & 31);
        fa[set][h][i] = *reinterpret_cast<const u32x4*>(at_a + h * TL::OPER + row * 128 + ((kg ^ swz64(row)) << 4));
      }
#pragma unroll
      for (int j = 0; j < TL::FN; ++j) {
        if constexpr (TRB) {
          const int k = sub * 16 + (lane >> 5) * 8 + ((lane & 15) >> 2);
          const int col = wj * TL::WTN + 32 * j + ((lane >> 4) & 1) * 16 + 4 * (lane & 3);
          typedef __attribute__((address_space(3))) s16x4* lptr;
          const char* p = at_b + h * TL::OPER + k * (2 * T) + (((col >> 3) ^ swz_down<T>(k)) << 4) + (col & 7) * 2;
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(p));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(p + 4 * (2 * T)));
          const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
          fb[set][h][j] = u32x4{l2[0], l2[1], h2[0], h2[1]};
        } else {
          const int row = wj * TL::WTN + 32 * j + (lane & 31);
          fb[set][h][j] = *reinterpret_cast<const u32x4*>(at_b + h * TL::OPER + row * 128 + ((kg ^ swz64(row)) << 4));
        }
      }
    }
  };
  // product n of a quarter of a step: the parts' three rounds over the accumulators, smallest terms first
  auto product = [&](auto nn, auto ss) {
    constexpr int n = decltype(nn)::value, set = decltype(ss)::value, i = n / TL::FN % TL::FM, j = n % TL::FN;
    constexpr int round = n / (TL::FM * TL::FN), ha = BOTH && round == 0, hb = BOTH && round == 1;
    acc[i][j] = ACROSS ? mfma_32x32x16<true>(fb[set][hb][j], fa[set][ha][i], acc[i][j])
                       : mfma_32x32x16<true>(fa[set][ha][i], fb[set][hb][j], acc[i][j]);
  };
  // the products of one quarter of a step with `count` loads, from `first` on, spread between them: issued in a row they
  // would hold the wave up until the memory path took them all
  auto products = [&](auto ss, auto first, auto count, auto&& load) {
    constexpr int N = TL::FM * TL::FN * (BOTH ? 3 : 1), F = decltype(first)::value, C = decltype(count)::value;
    static_for<N>([&](auto mm) {
      constexpr int m = decltype(mm)::value, before = m * C / N, after = (m + 1) * C / N;
      product(mm, ss);
      if constexpr (after > before) {
        __builtin_amdgcn_sched_barrier(0);
        static_for<after - before>([&](auto k) { load(std::integral_constant<int, F + before + decltype(k)::value>{}); });
        __builtin_amdgcn_sched_barrier(0);
      }
    });
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr std::integral_constant<int, 0> even{};
  constexpr std::integral_constant<int, 1> odd{};

  // Step i multiplies quarters 0 .. 3 of A(i), B(i), each from registers that were read during the quarter before.  The last
  // quarter comes behind the barrier that frees the tiles of step i and admits those of step i + 1, so no product
  // waits for the first operands of a step.  B(i + 2) is loaded right behind that barrier, A(i + 3) during the following
  // three quarters: the loads are spread over the step, and the ones issued late have a step more to arrive.
  constexpr int C0 = (LOADS + 1) / 2, C1 = (LOADS - C0 + 1) / 2, C2 = LOADS - C0 - C1;
  static_for<4>([&](auto u) {
    const Loads l = loads_of(decltype(u)::value / 2, decltype(u)::value % 2);
    static_for<LOADS>([&](auto j) {
      if constexpr (decltype(u)::value % 2) issue(l, vb, j);
      else issue(l, va, j);
    });
  });
  __builtin_amdgcn_s_waitcnt(vmcnt_only(2 * LOADS));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  fetch(0, 0, even);
  for (int i = 0; i < steps; ++i) {
    const Loads la = loads_of(i + 2, false), lb = loads_of(i + 2, true);
    auto from_a = [&](auto j) { issue(la, va, j); };
    fetch(i, 1, odd);
    __builtin_amdgcn_sched_barrier(0);
    products(even, std::integral_constant<int, 0>{}, std::integral_constant<int, C0>{}, from_a);
    fetch(i, 2, even);
    __builtin_amdgcn_sched_barrier(0);
    products(odd, std::integral_constant<int, C0>{}, std::integral_constant<int, C1>{}, from_a);
    fetch(i, 3, odd);
    __builtin_amdgcn_sched_barrier(0);
    products(even, std::integral_constant<int, C0 + C1>{}, std::integral_constant<int, C2>{}, from_a);
    // this wave's reads of step i are done, and all its loads but those of A(i + 2)
    __builtin_amdgcn_s_waitcnt(vmcnt_only(LOADS));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    fetch(i + 1, 0, even);                 // past the last step: what lies there, never used
    __builtin_amdgcn_sched_barrier(0);
    products(odd, std::integral_constant<int, 0>{}, std::integral_constant<int, LOADS>{}, [&](auto j) { issue(lb, vb, j); });
  }
  __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
}

// Writes a wave's tile of fp16 words 16 bytes a lane, with `mirror` the transpose too: 32 rows at a time through the
// wave's own part of LDS.  `value(i, j, v4, row, col, x)`: the four values of accumulator (i, j) from entry 4 v4 on, the
// first of them at row, col of the wave's tile; `ahead(i)` loads what they need for the accumulators i, 32 rows ahead.  Rows below `rows` and columns below `cols` are written, from `valid` on as zero.
template <class TL, int PARTS, class L, class V>
OD_DEV void ns_store(char* lds, L&& ahead, V&& value, uint16_t* out, int64_t plane, int ld, int row0, int col0, int rows, int cols,
                     int valid, bool mirror) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // 16-byte slots and bytes of a staged row, whose slots are rotated where they are a power of two, otherwise padded
  constexpr int SL = TL::WTN / 8, ROWB = SL * 16 + (SL & (SL - 1) ? 16 : 0), PIECE = 32 * ROWB;
  auto at = [](int r, int slot) { return r * ROWB + ((SL & (SL - 1) ? slot : slot ^ (SL == 8 ? swz64(r) : r & (SL - 1))) << 4); };
  static_assert(TL::NW * PARTS * PIECE <= TL::lds(PARTS), "staging");
  auto masked = [&](u32x4 w, int col) {
    if (col + 8 > valid) {
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] &= (col + 2 * k < valid ? 0xffffu : 0u) | (col + 2 * k + 1 < valid ? 0xffff0000u : 0u);
    }
    return w;
  };
  char* mine = lds + wave * (PARTS * PIECE);
  ahead(std::integral_constant<int, 0>{});
  static_for<TL::FM>([&](auto ii) {
    constexpr int i = decltype(ii)::value;
    if constexpr (i + 1 < TL::FM) ahead(std::integral_constant<int, i + 1>{});
    static_for<TL::FN * 4>([&](auto jj) {
      constexpr int j = decltype(jj)::value / 4, v4 = decltype(jj)::value % 4;
      const int r = lane & 31, c = 32 * j + 8 * v4 + 4 * (lane >> 5);
      float x[4];
      value(ii, std::integral_constant<int, j>{}, std::integral_constant<int, v4>{}, 32 * i + r, c, x);
      // both parts from one evaluation: evaluated once more, a value might be contracted differently, round to another
      // first word near a tie and leave a remainder of that one
      uint32_t a[PARTS], b[PARTS];
      split2<PARTS>(x[0], x[1], a);
      split2<PARTS>(x[2], x[3], b);
#pragma unroll
      for (int part = 0; part < PARTS; ++part)
        *reinterpret_cast<u32x2*>(mine + part * PIECE + at(r, c >> 3) + (c & 7) * 2) = u32x2{a[part], b[part]};
    });
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      uint16_t* o = out + part * plane;
      const char* piece = mine + part * PIECE;
#pragma unroll
      for (int it = 0; it < SL / 2; ++it) {
        const int r = (it * 64 + lane) / SL, slot = (it * 64 + lane) % SL;
        const u32x4 w = *reinterpret_cast<const u32x4*>(piece + at(r, slot));
        const int row = row0 + 32 * i + r, col = col0 + 8 * slot;
        if (row < rows && col < cols) *reinterpret_cast<u32x4*>(o + (int64_t)row * ld + col) = masked(w, col);
      }
      if (mirror) {
        // lane l receives rows 8 (l / 16) .. + 7 of column l % 16 of each block of 16 columns
        typedef __attribute__((address_space(3))) s16x4* lptr;
#pragma unroll
        for (int cb = 0; cb < TL::WTN / 16; ++cb) {
          const int c = cb * 16 + 4 * (lane & 3), r = (lane >> 4) * 8 + ((lane & 15) >> 2);
          const s16x4 h0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(piece + at(r, c >> 3) + (c & 7) * 2));
          const s16x4 h1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(piece + at(r + 4, c >> 3) + (c & 7) * 2));
          const u32x2 l2 = __builtin_bit_cast(u32x2, h0), h2 = __builtin_bit_cast(u32x2, h1);
          const int row = col0 + cb * 16 + (lane & 15), col = row0 + 32 * i + (lane >> 4) * 8;
          if (row < rows && col < cols) *reinterpret_cast<u32x4*>(o + (int64_t)row * ld + col) = masked(u32x4{l2[0], l2[1], h2[0], h2[1]}, col);
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  });
}

// tile of the upper triangle: row i holds tiles i .. n - 1
OD_DEV void upper_tile(int t, int n, int* ti, int* tj) {
  int i = 0;
  while (t >= n - i) {
    t -= n - i;
    ++i;
  }
  *ti = i;
  *tj = i + t;
}

// The jobs of one launch.
template <class TL, int PARTS>
__global__ __launch_bounds__(TL::THREADS, TL::blocks(PARTS)) void k_ns_products(NsArgs args) {
  extern __shared__ __align__(16) char lds[];
  constexpr int T = TL::T;
  const int bid = xcd_contiguous(blockIdx.x, args.total);
  const NsJob c = args.j[ns_job(args, bid)];
  const int pp = up64(c.p), qq = up64(c.q), ni = (c.p + T - 1) / T, local = bid - c.first;
  const int64_t yplane = (int64_t)pp * c.lq, splane = (int64_t)c.p * c.lp;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  f32x16 acc[TL::FM][TL::FN];
  const int kind = __builtin_amdgcn_readfirstlane(c.kind);       // a scalar branch: the loads below set the lane mask
  if (kind == NS_APPLY) {
    const int nj = (c.q + T - 1) / T;
    const int z = quotient(local, ni * nj), tl = local - z * (ni * nj);
    const int tj = quotient(tl, ni), ti = tl - tj * ni;
    uint16_t* slice = c.base + z * c.stride;
    const NsOperand A{slice + c.a + (int64_t)ti * T * c.lp, splane, c.lp, c.p - ti * T}, B{slice + c.b + tj * T, yplane, c.lq, qq - tj * T};
    ns_product<TL, PARTS, true, true>(acc, A, B, pp, lds);
    __syncthreads();
    const int row0 = ti * T + wave / TL::WJ * TL::WTM, col0 = tj * T + wave % TL::WJ * TL::WTN;
    ns_store<TL, PARTS>(lds, [](auto) {}, [&](auto i, auto j, auto v4, int, int, float* x) {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = c.cc * acc[i][j][4 * v4 + e];
    }, slice + c.out, yplane, c.lq, row0, col0, c.p, qq, c.q, false);
  } else {
    const bool full = kind == NS_FULL;
    const int splits = c.splits > 0 ? c.splits : 1, tiles = full ? ni * ni : ni * (ni + 1) / 2, per = tiles * splits;
    const int z = quotient(local, per), in_z = local - z * per, tile = quotient(in_z, splits), split = in_z - tile * splits;
    int ti, tj;
    if (full) {
      tj = quotient(tile, ni);
      ti = tile - tj * ni;
    } else {
      upper_tile(tile, ni, &ti, &tj);
    }
    uint16_t* slice = c.base + z * c.stride;
    const bool gram = kind == NS_GRAM;
    const int64_t plane = gram ? yplane : splane;
    const int ld = gram ? c.lq : c.lp;
    const NsOperand A{slice + c.a + (int64_t)ti * T * ld, plane, ld, c.p - ti * T}, B{slice + c.b + (int64_t)tj * T * ld, plane, ld, c.p - tj * T};
    ns_product<TL, PARTS, false, true>(acc, A, B, gram ? qq : pp, lds, split, splits);
    if (c.splits > 0) {
      const int lane = threadIdx.x & 63;
      float* out = reinterpret_cast<float*>(slice + c.out) + (int64_t)in_z * T * T;
      static_for<TL::FM * TL::FN * 4>([&](auto n) {
        constexpr int i = decltype(n)::value / (4 * TL::FN), j = decltype(n)::value / 4 % TL::FN, v4 = decltype(n)::value % 4;
        const int r = wave / TL::WJ * TL::WTM + 32 * i + (lane & 31), cl = wave % TL::WJ * TL::WTN + 32 * j + 8 * v4 + 4 * (lane >> 5);
        *reinterpret_cast<f32x4*>(out + r * T + cl) = f32x4{acc[i][j][4 * v4], acc[i][j][4 * v4 + 1], acc[i][j][4 * v4 + 2], acc[i][j][4 * v4 + 3]};
      });
      return;
    }
    __syncthreads();
    const int row0 = ti * T + wave / TL::WJ * TL::WTM, col0 = tj * T + wave % TL::WJ * TL::WTN;
    const uint16_t* E = slice + c.e;
    const int lane = threadIdx.x & 63;
    u32x2 word[2][PARTS][TL::FN][4];             // of e, for two blocks of 32 rows
    ns_store<TL, PARTS>(lds, [&](auto i) {
      constexpr int set = decltype(i)::value & 1;
      const int row = min(row0 + 32 * i + (lane & 31), c.p - 1);
      if (c.cb == 0.f) return;
#pragma unroll
      for (int part = 0; part < PARTS; ++part)
#pragma unroll
        for (int j = 0; j < TL::FN; ++j)
#pragma unroll
          for (int v4 = 0; v4 < 4; ++v4)
            word[set][part][j][v4] = *reinterpret_cast<const u32x2*>(E + part * splane + (int64_t)row * c.lp + min(col0 + 32 * j + 8 * v4 + 4 * (lane >> 5), pp - 4));
    }, [&](auto i, auto j, auto v4, int r, int cl, float* x) {
      const int row = row0 + r, col = col0 + cl;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = c.cc * acc[i][j][4 * v4 + e] + (row == col + e ? c.ca : 0.f);
      if (c.cb != 0.f) {
#pragma unroll
        for (int part = 0; part < PARTS; ++part)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t pair = word[i & 1][part][j][v4][e];      // a bit cast of a vector's element itself would take its first one
            const f16x2 h = __builtin_bit_cast(f16x2, pair);
            x[2 * e] += c.cb * (float)h[0];
            x[2 * e + 1] += c.cb * (float)h[1];
          }
      }
    }, slice + c.out, splane, c.lp, row0, col0, c.p, pp, c.p, !full && ti != tj);
  }
}

// Adds the partial sums of a Gram matrix in their order: one workgroup 8 rows of a tile, written in both triangles.
// Bound by the latency of the loads, four of them in flight.
template <int PARTS>
__global__ __launch_bounds__(256) void k_ns_reduce(NsArgs args) {
  constexpr int T = kNsSplitTile, R = 8;
  __shared__ float tile[R][T + 4];
  const NsJob c = args.j[ns_job(args, blockIdx.x)];
  const int pp = up64(c.p), n = (c.p + T - 1) / T, tiles = n * (n + 1) / 2, local = blockIdx.x - c.first;
  const int z = quotient(local, T / R * tiles), in_z = local - z * (T / R) * tiles, t = in_z / (T / R), r0 = in_z % (T / R) * R;
  int ti, tj;
  upper_tile(t, n, &ti, &tj);
  if (ti * T + r0 >= c.p) return;
  uint16_t* slice = c.base + z * c.stride;
  const int64_t splane = (int64_t)c.p * c.lp;
  const int tid = threadIdx.x, r = tid >> 5, c0 = (tid & 31) * 4;
  const float* in = reinterpret_cast<const float*>(slice + c.a) + (int64_t)t * c.splits * T * T + (r0 + r) * T + c0;
  f32x4 sum = {};
#pragma unroll 4
  for (int s = 0; s < c.splits; ++s) sum += *reinterpret_cast<const f32x4*>(in + (int64_t)s * T * T);
#pragma unroll
  for (int e = 0; e < 4; ++e) tile[r][c0 + e] = c.cc * sum[e];
  __syncthreads();
  uint16_t* out = slice + c.out;
  auto put = [&](int row, int col, auto&& at) {
    u32x4 w[PARTS];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t s[PARTS];
      split2<PARTS>(col + 2 * e < c.p ? at(2 * e) : 0.f, col + 2 * e + 1 < c.p ? at(2 * e + 1) : 0.f, s);
#pragma unroll
      for (int part = 0; part < PARTS; ++part) w[part][e] = s[part];
    }
#pragma unroll
    for (int part = 0; part < PARTS; ++part) *reinterpret_cast<u32x4*>(out + part * splane + (int64_t)row * c.lp + col) = w[part];
  };
  // eight columns of a row a thread; above the diagonal also eight rows of a column, all of them inside
  if (tid < R * (T / 8)) {
    const int k = tid / (T / 8), row = ti * T + r0 + k, col = tj * T + tid % (T / 8) * 8;
    if (row < c.p && col < pp) put(row, col, [&](int e) { return tile[k][tid % (T / 8) * 8 + e]; });
  } else if (ti != tj) {
    const int k = tid - R * (T / 8), row = tj * T + k;
    if (row < c.p) put(row, ti * T + r0, [&](int e) { return tile[e][k]; });
  }
}

// All p x p work of a segment of steps for one matrix of p <= D, in one workgroup, with the Gram matrix before it where Y fits into
// LDS: S and P lie in LDS as two fp16 words a
// value (22 bits, three products), T = P S and Z in the accumulators' registers, from where they change places with S.
// A wave has one 32 x 32 block.  A chain of products with a barrier after each: bound by the latency of LDS and barriers.
template <int D>
struct NsSmallTile {
  static constexpr int W = D / 32, THREADS = 64 * W * W;
  static constexpr int PITCH = D * 2 + 16, PLANE = D * PITCH;      // an odd number of 16-byte slots: rows in different banks
  static constexpr int lds(int) { return 4 * PLANE; }
};

template <int D, int PARTS>
__global__ __launch_bounds__(NsSmallTile<D>::THREADS, 1) void k_ns_small(NsJobs<kNsClasses> args, NsSteps k) {
  typedef NsSmallTile<D> TL;
  extern __shared__ __align__(16) char lds[];
  const NsJob c = args.j[ns_job(args, blockIdx.x)];
  const int z = blockIdx.x - c.first, pp = up64(c.p);
  uint16_t* slice = c.base + z * c.stride;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // entry n of the accumulator: row `row`, column col0 + 8 (n / 4) + n % 4
  const int row = wave / TL::W * 32 + (lane & 31), block = wave % TL::W * 32, col0 = block + 4 * (lane >> 5);
  char* const s_plane = lds;
  char* const p_plane = lds + 2 * TL::PLANE;
  auto product = [&](const char* a, const char* b) {
    f32x16 hh, rest;
#pragma unroll
    for (int n = 0; n < 16; ++n) hh[n] = rest[n] = 0.f;
    const char* pa = a + row * TL::PITCH + (lane >> 5) * 16;
    const char* pb = b + (block + (lane & 31)) * TL::PITCH + (lane >> 5) * 16;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const u32x4 ah = *reinterpret_cast<const u32x4*>(pa + 32 * ks), al = *reinterpret_cast<const u32x4*>(pa + TL::PLANE + 32 * ks);
      const u32x4 bh = *reinterpret_cast<const u32x4*>(pb + 32 * ks), bl = *reinterpret_cast<const u32x4*>(pb + TL::PLANE + 32 * ks);
      hh = mfma_32x32x16<true>(bh, ah, hh);
      rest = mfma_32x32x16<true>(bl, ah, rest);
      rest = mfma_32x32x16<true>(bh, al, rest);
    }
    return hh + rest;
  };
  auto put = [&](char* plane, const f32x16& v, float scale) {
#pragma unroll
    for (int v4 = 0; v4 < 4; ++v4) {
      uint32_t a[2], b[2];
      split2<2>(scale * v[4 * v4], scale * v[4 * v4 + 1], a);
      split2<2>(scale * v[4 * v4 + 2], scale * v[4 * v4 + 3], b);
#pragma unroll
      for (int part = 0; part < 2; ++part)
        *reinterpret_cast<u32x2*>(plane + part * TL::PLANE + row * TL::PITCH + (col0 + 8 * v4) * 2) = u32x2{a[part], b[part]};
    }
  };
  // S, zero outside the matrix
  f32x16 s, p, zz, t;
#pragma unroll
  for (int n = 0; n < 16; ++n) s[n] = 0.f;
  if (c.splits == 0) {
    // from Y, all of which fits where S and P will lie (ns_small_whole): at most eight 16-byte groups a thread, all in flight
    const int qq = up64(c.q), slots = qq / 8, pitch = qq * 2 + 16, all = D * slots, most = PARTS * all;
    const int64_t yplane = (int64_t)pp * c.lq;
    const uint16_t* y = slice + c.a;
    u32x4 w[8];
    int at[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int n = min((int)threadIdx.x + i * TL::THREADS, most - 1), part = n >= all, r = (n - part * all) / slots, slot = n - part * all - r * slots;
      w[i] = *reinterpret_cast<const u32x4*>(y + part * yplane + (int64_t)r * c.lq + slot * 8);
      at[i] = (part * D + r) * pitch + slot * 16;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<u32x4*>(lds + at[i]) = w[i];
    __syncthreads();
    f32x16 rest;
#pragma unroll
    for (int n = 0; n < 16; ++n) rest[n] = 0.f;
    const char* pa = lds + row * pitch + (lane >> 5) * 16;
    const char* pb = lds + (block + (lane & 31)) * pitch + (lane >> 5) * 16;
#pragma unroll 4
    for (int ks = 0; ks < qq / 16; ++ks) {
      const u32x4 ah = *reinterpret_cast<const u32x4*>(pa + 32 * ks), bh = *reinterpret_cast<const u32x4*>(pb + 32 * ks);
      s = mfma_32x32x16<true>(bh, ah, s);
      if constexpr (PARTS == 2) {
        const u32x4 al = *reinterpret_cast<const u32x4*>(pa + D * pitch + 32 * ks), bl = *reinterpret_cast<const u32x4*>(pb + D * pitch + 32 * ks);
        rest = mfma_32x32x16<true>(bl, ah, rest);
        rest = mfma_32x32x16<true>(bh, al, rest);
      }
    }
    s += rest;
    __syncthreads();
  } else {
    const float* in = reinterpret_cast<const float*>(slice + c.a) + row * kNsSplitTile + col0;
#pragma unroll 4
    for (int split = 0; split < c.splits; ++split)
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(in + (int64_t)split * kNsSplitTile * kNsSplitTile + 8 * v4);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * v4 + e] += x[e];
      }
  }
#pragma unroll
  for (int n = 0; n < 16; ++n) s[n] = row < c.p && col0 + 8 * (n >> 2) + (n & 3) < c.p ? c.cc * s[n] : 0.f;
  for (int l = 0; l < k.count; ++l) {
    if (l > 0) {
      t = product(p_plane, s_plane) * (1.f / (k.p[l - 1] * k.s[l - 1]));            // T = P S
      __syncthreads();
      if (l > 1) {
        put(s_plane, zz, k.z[l - 2]);
        __syncthreads();
        zz = product(p_plane, s_plane) * (1.f / (k.p[l - 1] * k.z[l - 2]));         // Z = P Z
        __syncthreads();
      } else {
        zz = p;
      }
      put(s_plane, t, k.t[l - 1]);
      __syncthreads();
      s = product(s_plane, p_plane) * (1.f / (k.t[l - 1] * k.p[l - 1]));            // S = T P
      __syncthreads();
    }
    put(s_plane, s, k.s[l]);
    __syncthreads();
    p = product(s_plane, s_plane) * (k.c[l] / (k.s[l] * k.s[l]));                   // P = a I + b S + c S S
#pragma unroll
    for (int n = 0; n < 16; ++n) p[n] += k.b[l] * s[n] + (row == col0 + 8 * (n >> 2) + (n & 3) && row < c.p ? k.a[l] : 0.f);
    put(p_plane, p, k.p[l]);
    __syncthreads();
  }
  if (k.count > 1) {
    put(s_plane, zz, k.z[k.count - 2]);
    __syncthreads();
    p = product(p_plane, s_plane) * (1.f / (k.p[k.count - 1] * k.z[k.count - 2]));  // Z = P Z
  }
  // Z out, rows of pp columns
  const int64_t splane = (int64_t)c.p * c.lp;
#pragma unroll
  for (int v4 = 0; v4 < 4; ++v4) {
    const int col = col0 + 8 * v4;
    uint32_t a[PARTS], b[PARTS];
    const float f = k.z[k.count - 1];
    split2<PARTS>(f * p[4 * v4], f * p[4 * v4 + 1], a);
    split2<PARTS>(f * p[4 * v4 + 2], f * p[4 * v4 + 3], b);
    if (row < c.p) {
#pragma unroll
      for (int part = 0; part < PARTS; ++part) *reinterpret_cast<u32x2*>(slice + c.out + part * splane + (int64_t)row * c.lp + col) = u32x2{a[part], b[part]};
    }
  }
  // columns D .. pp, which no block holds
  for (int n = threadIdx.x; n < c.p * ((pp - D) / 8); n += TL::THREADS) {
    const int r = n / ((pp - D) / 8), slot = n % ((pp - D) / 8);
#pragma unroll
    for (int part = 0; part < PARTS; ++part) *reinterpret_cast<u32x4*>(slice + c.out + part * splane + (int64_t)r * c.lp + D + 8 * slot) = u32x4{0u, 0u, 0u, 0u};
  }
}

// O = P Y into the caller's matrix, or its update.  TALL: the accumulators lie the other way round, so that either way a lane
// has four consecutive columns of a row of the caller's matrix.
template <class TL, int PARTS, bool XBF, bool TALL>
OD_DEV void ns_final_tile(const NsJob& c, int z, int ti, int tj, const MuonTables& t, int update, float keep, float lr, char* lds) {
  constexpr int T = TL::T;
  const float scale = c.cc;
  const int pp = up64(c.p), qq = up64(c.q);
  const int64_t yplane = (int64_t)pp * c.lq, splane = (int64_t)c.p * c.lp;
  uint16_t* slice = c.base + z * c.stride;
  const NsOperand A{slice + c.a + (int64_t)ti * T * c.lp, splane, c.lp, c.p - ti * T}, B{slice + c.b + tj * T, yplane, c.lq, qq - tj * T};
  f32x16 acc[TL::FM][TL::FN];
  ns_product<TL, PARTS, true, !TALL>(acc, A, B, pp, lds);
  const MuonMat a = t.mats[c.mat0 + z];
  const MuonEntry e = t.entries[c.mat0 + z];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i0 = ti * T + wave / TL::WJ * TL::WTM, j0 = tj * T + wave % TL::WJ * TL::WTN;
  const bool vec = rows_aligned(e.X, a.ldx);
  const float step = update ? lr * a.scale * scale : -scale;
  const float kx = update ? keep : 0.f;
  // 32 rows of the matrix at a time through the wave's own part of LDS, from where a lane takes eight columns of a row
  constexpr int COLS = TALL ? TL::WTM : TL::WTN, PITCH = COLS * 4 + 16, GROUPS = COLS / 8;
  static_assert(TL::NW * 32 * PITCH <= TL::lds(PARTS), "staging");
  char* mine = lds + wave * (32 * PITCH);
  __syncthreads();
  static_for<TALL ? TL::FN : TL::FM>([&](auto bb) {
    constexpr int blk = decltype(bb)::value;
    static_for<COLS / 32 * 4>([&](auto n) {
      constexpr int c = decltype(n)::value / 4, v4 = decltype(n)::value % 4;
      const f32x16& v = acc[TALL ? c : blk][TALL ? blk : c];
      *reinterpret_cast<f32x4*>(mine + (lane & 31) * PITCH + (32 * c + 8 * v4 + 4 * (lane >> 5)) * 4) = f32x4{v[4 * v4], v[4 * v4 + 1], v[4 * v4 + 2], v[4 * v4 + 3]};
    });
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int it = 0; it < GROUPS / 2; ++it) {
      const int k = it * 64 + lane, r = k / GROUPS, g = k % GROUPS;
      const int row = (TALL ? j0 : i0) + 32 * blk + r, col = (TALL ? i0 : j0) + 8 * g;
      if (row >= a.m || col >= a.n) continue;
      const f32x4* o = reinterpret_cast<const f32x4*>(mine + r * PITCH + g * 32);
      const f32x4 o0 = o[0], o1 = o[1];
      const int64_t at = (int64_t)row * a.ldx + col;
      float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      const bool whole = vec && col + 8 <= a.n;
      if (update) {
        if (whole) load8<XBF>(e.X, at, x);
        else {
#pragma unroll
          for (int q = 0; q < 8; ++q) x[q] = load_elem<XBF>(e.X, at + min(q, a.n - 1 - col));      // all in flight, no branch
        }
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] = kx * x[q] - step * (q < 4 ? o0[q & 3] : o1[q & 3]);
      if (whole) {
        if constexpr (XBF) {
          *reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(e.X) + at) = u32x4{pack_bf16_rne(x[0], x[1]), pack_bf16_rne(x[2], x[3]), pack_bf16_rne(x[4], x[5]), pack_bf16_rne(x[6], x[7])};
        } else {
          f32x4* px = reinterpret_cast<f32x4*>(reinterpret_cast<float*>(e.X) + at);
          px[0] = f32x4{x[0], x[1], x[2], x[3]};
          px[1] = f32x4{x[4], x[5], x[6], x[7]};
        }
      } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          if (col + q >= a.n) continue;
          if constexpr (XBF) reinterpret_cast<uint16_t*>(e.X)[at + q] = (uint16_t)pack_bf16_rne(x[q], 0.f);
          else reinterpret_cast<float*>(e.X)[at + q] = x[q];
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  });
}

template <class TL, int PARTS, bool XBF>
__global__ __launch_bounds__(TL::THREADS, TL::blocks(PARTS)) void k_ns_final(NsArgs args, MuonTables t, int update, float keep, float lr) {
  extern __shared__ __align__(16) char lds[];
  const int bid = xcd_contiguous(blockIdx.x, args.total);
  const NsJob c = args.j[ns_job(args, bid)];
  const int ni = (c.p + TL::T - 1) / TL::T, nj = (c.q + TL::T - 1) / TL::T, local = bid - c.first;
  const int z = quotient(local, ni * nj), tl = local - z * (ni * nj);
  const int tj = quotient(tl, ni), ti = tl - tj * ni;
  if (__builtin_amdgcn_readfirstlane(c.tall)) ns_final_tile<TL, PARTS, XBF, true>(c, z, ti, tj, t, update, keep, lr, lds);
  else ns_final_tile<TL, PARTS, XBF, false>(c, z, ti, tj, t, update, keep, lr, lds);
}

// ------------------------------------------------------------------------------------
// Launchers
// ------------------------------------------------------------------------------------
hipError_t launch_muon_begin(const MuonEntry* entries, const MuonMat* mats, int mat0, int count, const MuonTables& t, float mu,
                             bool nesterov, bool g_bf16, hipStream_t st) {
  for (int k = 0; k < count; k += kMuonChunk) {
    MuonChunk chunk = {};
    const int n = count - k < kMuonChunk ? count - k : kMuonChunk;
    int blocks = 1;
    for (int i = 0; i < n; ++i) {
      chunk.e[i] = entries[k + i];
      chunk.m[i] = mats[k + i];
      blocks = mats[k + i].blocks > blocks ? mats[k + i].blocks : blocks;
    }
    const dim3 grid(blocks, n);
    if (g_bf16) k_muon_begin<true><<<grid, 256, 0, st>>>(chunk, t, mat0 + k, mu, nesterov);
    else k_muon_begin<false><<<grid, 256, 0, st>>>(chunk, t, mat0 + k, mu, nesterov);
    const hipError_t rc = hipGetLastError();
    if (rc != hipSuccess) return rc;
  }
  return hipSuccess;
}

namespace {

// the jobs that `take` accepts, with the workgroups that `tiles` gives per matrix
template <int N = kNsJobs, class Take, class Tiles>
NsJobs<N> laid_out(const NsArgs& a, Take&& take, Tiles&& tiles) {
  NsJobs<N> o;
  o.count = o.total = 0;
  for (int k = 0; k < a.count; ++k) {
    if (!take(a.j[k])) continue;
    o.j[o.count] = a.j[k];
    o.j[o.count++].first = o.total;
    o.total += a.j[k].nb * tiles(a.j[k]);
  }
  return o;
}

int ceil_div(int a, int b) { return (a + b - 1) / b; }
bool any(const NsJob&) { return true; }

// more than 64 KB of LDS have to be asked for
template <class K>
hipError_t allow_lds(K* kernel, int bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <class TL, int PARTS, class K, int N, class... A>
hipError_t go(K* kernel, const NsJobs<N>& a, hipStream_t st, A... rest) {
  if (a.total == 0) return hipSuccess;
  const hipError_t rc = allow_lds(kernel, TL::lds(PARTS));
  if (rc != hipSuccess) return rc;
  kernel<<<a.total, TL::THREADS, TL::lds(PARTS), st>>>(a, rest...);
  return hipGetLastError();
}

typedef NsTile<64, 2, 2> Tiny;
typedef NsTile<128, 2, 2> Small;
typedef NsTile<192, 2, 2> Mid;
typedef NsTile<256, 2, 4> Large;
static_assert(Small::T == kNsSplitTile, "partial sums are those of its tiles");

template <int T>
int tiles_of(const NsJob& c) {
  const int n = ceil_div(c.p, T);
  return c.kind == NS_APPLY ? n * ceil_div(c.q, T) : c.kind == NS_FULL ? n * n : n * (n + 1) / 2 * (c.splits > 0 ? c.splits : 1);
}

}  // namespace

// The tile for these jobs: the one with the least time in us by what a step of 64 k and a workgroup's beginning and
// end take.  256 CUs; beyond one round of workgroups the last one counts half by what is in it, half as a whole one.
// One word: 64 x 64 0.43 a step, 0.30 for each workgroup of a CU where there are more, and 4; 128 x 128 0.7 and 4 alone on a CU, 1.0
// and 5 for two side by side, 1.2 where that happens everywhere and the clock gives way; 192 x 192 1.15 and 6, 1.43 in several
// rounds; 256 x 256 1.7 and 8, 1.85 with most CUs at work.
// Two words: 64 x 64 0.8 and 0.65, 128 x 128 1.7 a round (one workgroup fits a CU), 256 x 256 5.2 and 6.3 (three passes).
// Measured on products of 264 x 264 to 4096 x 4096, 1 to 72 matrices: the rule takes the fastest or one within 10 %.
int ns_tile(const NsArgs& a, int parts) {
  double n64 = 0.0, n128 = 0.0, n192 = 0.0, n256 = 0.0, steps = 0.0;
  for (int k = 0; k < a.count; ++k) {
    const NsJob& j = a.j[k];
    if (j.splits > 0) return Small::T;                 // partial sums
    const double nb = j.nb, n = nb * tiles_of<256>(j);
    n64 += nb * tiles_of<64>(j);
    n128 += nb * tiles_of<128>(j);
    n192 += nb * tiles_of<192>(j);
    n256 += n;
    steps += n * ceil_div(j.kind == NS_GRAM ? j.q : j.p, kNsStep);
  }
  const double s = steps / n256, pairs = std::floor(n128 / 512.0), rest = n128 - 512.0 * pairs;
  auto rounds = [](double n) { return n <= 256.0 ? 1.0 : 0.5 * n / 256.0 + 0.5 * std::ceil(n / 256.0) + 0.15; };
  double t64, t128, t192, t256;
  if (parts == 1) {
    t64 = std::max(0.43, 0.30 / 256.0 * n64) * s + 4.0;
    t128 = pairs * (1.2 * s + 5.0) + (rest == 0.0 ? 0.0 : rest <= 256.0 ? 0.7 * s + 4.0 : 1.0 * s + 5.0);
    t192 = rounds(n192) * ((n192 <= 256.0 ? 1.15 : 1.43) * s + 6.0);
    t256 = rounds(n256) * ((n256 < 200.0 ? 1.7 : 1.85) * s + 8.0);
  } else {
    t64 = std::max(0.8, 0.65 / 256.0 * n64) * s + 4.0;
    t128 = std::ceil(n128 / 256.0) * (1.7 * s + 5.0);
    t192 = INFINITY;
    t256 = std::ceil(n256 / 256.0) * ((n256 < 200.0 ? 5.2 : 6.3) * s + 8.0);
  }
  t192 *= 1.07;                                        // the least even of the four: taken where it is clearly ahead
  const double least = std::min(std::min(t64, t128), std::min(t192, t256));
  return least == t64 ? Tiny::T : least == t128 ? Small::T : least == t192 ? Mid::T : Large::T;
}

namespace {

// f with that tile
template <class F>
hipError_t with_tile(const NsArgs& a, int parts, F&& f) {
  switch (ns_tile(a, parts)) {
    case Tiny::T: return f(Tiny{});
    case Small::T: return f(Small{});
    case Mid::T: return f(Mid{});
    default: return f(Large{});
  }
}

template <class TL, int PARTS, bool XBF>
hipError_t final_of(const NsArgs& a, const MuonTables& t, bool update, float keep, float lr, hipStream_t st) {
  return go<TL, PARTS>(k_ns_final<TL, PARTS, XBF>, laid_out(a, any, tiles_of<TL::T>), st, t, (int)update, keep, lr);
}

template <class TL>
hipError_t products_of(const NsArgs& a, int parts, hipStream_t st) {
  const NsArgs o = laid_out(a, any, tiles_of<TL::T>);
  if constexpr (TL::T != 192) {
    if (parts == 2) return go<TL, 2>(k_ns_products<TL, 2>, o, st);
  }
  return go<TL, 1>(k_ns_products<TL, 1>, o, st);
}

template <class TL>
hipError_t final_tiles(const NsArgs& a, const MuonTables& t, int parts, bool update, float keep, float lr, bool x_bf16, hipStream_t st) {
  if constexpr (TL::T != 192) {
    if (parts == 2) return x_bf16 ? final_of<TL, 2, true>(a, t, update, keep, lr, st) : final_of<TL, 2, false>(a, t, update, keep, lr, st);
  }
  return x_bf16 ? final_of<TL, 1, true>(a, t, update, keep, lr, st) : final_of<TL, 1, false>(a, t, update, keep, lr, st);
}

}  // namespace

hipError_t launch_muon_scale(const NsArgs& a, const MuonTables& t, float mu, bool nesterov, bool g_bf16, int parts, double eps,
                             double scale, hipStream_t st) {
  const NsArgs o = laid_out(a, any, [](const NsJob& c) { return ceil_div(c.p, 64) * ceil_div(c.q, 64); });
  auto run = [&](auto kernel) { kernel<<<o.total, 256, 0, st>>>(o, t, mu, (int)nesterov, eps, scale); };
  if (g_bf16) parts == 2 ? run(k_muon_scale<true, 2>) : run(k_muon_scale<true, 1>);
  else parts == 2 ? run(k_muon_scale<false, 2>) : run(k_muon_scale<false, 1>);
  return hipGetLastError();
}

hipError_t launch_ns_products(const NsArgs& a, int parts, hipStream_t st) {
  return with_tile(a, parts, [&](auto tile) { return products_of<decltype(tile)>(a, parts, st); });
}

hipError_t launch_ns_reduce(const NsArgs& a, int parts, hipStream_t st) {
  const NsArgs o = laid_out(a, any, [](const NsJob& c) { const int n = ceil_div(c.p, kNsSplitTile); return kNsSplitTile / 8 * (n * (n + 1) / 2); });
  if (parts == 2) k_ns_reduce<2><<<o.total, 256, 0, st>>>(o);
  else k_ns_reduce<1><<<o.total, 256, 0, st>>>(o);
  return hipGetLastError();
}

namespace {

template <int D, int PARTS>
hipError_t small_of(const NsArgs& a, const NsSteps& steps, hipStream_t st) {
  const NsJobs<kNsClasses> o = laid_out<kNsClasses>(a, [](const NsJob& c) { return ns_small_size(c.p) == D; }, [](const NsJob&) { return 1; });
  return go<NsSmallTile<D>, PARTS>(k_ns_small<D, PARTS>, o, st, steps);
}

template <int PARTS>
hipError_t small_sizes(const NsArgs& a, const NsSteps& steps, hipStream_t st) {
  hipError_t rc = small_of<32, PARTS>(a, steps, st);
  if (rc == hipSuccess) rc = small_of<64, PARTS>(a, steps, st);
  if (rc == hipSuccess) rc = small_of<96, PARTS>(a, steps, st);
  if (rc == hipSuccess) rc = small_of<128, PARTS>(a, steps, st);
  return rc;
}

}  // namespace

hipError_t launch_ns_small(const NsArgs& a, const NsSteps& steps, int parts, hipStream_t st) {
  return parts == 2 ? small_sizes<2>(a, steps, st) : small_sizes<1>(a, steps, st);
}

hipError_t launch_ns_final(const NsArgs& a, const MuonTables& t, int parts, bool update, float keep, float lr, bool x_bf16, hipStream_t st) {
  return with_tile(a, parts, [&](auto tile) { return final_tiles<decltype(tile)>(a, t, parts, update, keep, lr, x_bf16, st); });
}

}  // namespace od
