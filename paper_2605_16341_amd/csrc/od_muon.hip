// Muon: Newton-Schulz orthogonalisation of a set of matrices and the optimizer step around it (the method's
// published form: quintic iteration on the Frobenius-normalised momentum).  For every matrix
//   M  = mu M + G,   B = G + mu M (Nesterov) or M
//   X0 = B / (||B||_F + eps)
//   S  = Xk Xk^T,   P = a I + b S + c S S,   Xk+1 = P Xk        K times
//   X  = (1 - lr wd) X - lr scale XK
// S, S S and P are symmetric: only tiles on and above the diagonal are computed, the others mirrored.
// See od_muon.h for the layout of the workspace.
#include "od_muon.h"

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

// One workgroup: a range of rows of one matrix.  HBM bound: G read, M read and written.
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
  const int64_t rows = ((int64_t)a.m + a.blocks - 1) / a.blocks;
  const int64_t r0 = blockIdx.x * rows, r1 = min((int64_t)a.m, r0 + rows);
  double sum = 0.0;
  const bool vec = rows_aligned(e.G, a.ldg) && (e.M == nullptr || rows_aligned(e.M, a.ldm));
  // threads side by side along a row: the power of two at or above its items, so that narrow rows share a wave
  const int wide = vec ? a.n / 8 : 0;                       // whole groups of eight
  auto spread = [](int items) { int s = 1; while (s < 256 && s < items) s <<= 1; return s; };
  if (wide > 0) {
    const int tx = spread(wide), x = threadIdx.x & (tx - 1), y = threadIdx.x / tx, ty = 256 / tx;
    for (int64_t r = r0 + y; r < r1; r += ty)
      for (int c = x; c < wide; c += tx) {
        float g[8];
        load8<GBF>(e.G, r * a.ldg + 8 * c, g);
        if (e.M) {
          float m[8];
          f32x4* mp = reinterpret_cast<f32x4*>(e.M + r * a.ldm + 8 * c);
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
  const int c0 = 8 * wide, rest = a.n - c0;
  if (rest > 0) {
    const int tx = spread(rest), x = threadIdx.x & (tx - 1), y = threadIdx.x / tx, ty = 256 / tx;
    for (int64_t r = r0 + y; r < r1; r += ty)
      for (int c = c0 + x; c < a.n; c += tx) {
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

OD_DEV int ns_class(const NsArgs& a, int bid) {
  int k = 0;
  while (k + 1 < a.nclass && bid >= a.c[k + 1].first) ++k;
  return k;
}

OD_DEV int up64(int v) { return (v + 63) & ~63; }

// One workgroup: a 64 x 64 tile of Y (transposed on the way through LDS where the matrix is tall).  HBM bound.
template <bool GBF, int PARTS>
__global__ __launch_bounds__(256) void k_muon_scale(NsArgs args, MuonTables t, float mu, int nesterov, double eps, double scale) {
  __shared__ double lds[4];
  __shared__ float tile[64][65];
  const NsClass c = args.c[ns_class(args, blockIdx.x)];
  const int pp = up64(c.p), qq = up64(c.q), ti_n = pp / 64, tj_n = qq / 64;
  const int in_class = blockIdx.x - c.first, z = in_class / (ti_n * tj_n), tl = in_class % (ti_n * tj_n);
  const int ti = tl / tj_n, tj = tl % tj_n;
  const MuonMat a = t.mats[c.mat0 + z];
  const MuonEntry e = t.entries[c.mat0 + z];
  const int tid = threadIdx.x;
  double part = tid < a.blocks ? t.partials[(int64_t)(c.mat0 + z) * kMuonParts + tid] : 0.0;
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
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        b[i] = 0.f;
        if (r < a.m && cc + i < a.n) {
          b[i] = load_elem<GBF>(e.G, (int64_t)r * a.ldg + cc + i);
          if (e.M) {
            const float m = e.M[(int64_t)r * a.ldm + cc + i];
            b[i] = nesterov ? b[i] + mu * m : m;
          }
        }
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
// operands come by direct-to-LDS loads into two stages:
//   k along rows   128-byte rows, their 16-byte k-groups XOR-swizzled by (row >> 1) & 7: the 16 lanes that a
//                  ds_read_b128 serves at a time lie in 16 different groups of four banks
//   k down columns rows of T elements, their 64-byte blocks XOR-swizzled by k & 3, so that the four rows of a
//                  ds_read_b64_tr_b16 lie in different banks
// With two parts a product is three passes over K: hi hi, hi lo, lo hi.
// ------------------------------------------------------------------------------------
OD_DEV void dma16_at(uint32_t voff, const void* sbase, uint32_t lds_base) {
  const uint32_t l = __builtin_amdgcn_readfirstlane(lds_base);
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1\n" ::"v"(voff), "s"(sbase), "s"(l) : "memory");
}

OD_DEV int swz64(int row) { return (row >> 1) & 7; }

struct NsOperand {
  const uint16_t* p;      // tile's first row (TRB: the tile's first column is in `edge`)
  int64_t plane;          // elements between parts
  int ld;
  int rows;               // rows (TRB: columns) from the tile's first one that may be read, at least 1 (TRB: 8)
};

template <int T_, int WI_, int WJ_>
struct NsTile {
  static constexpr int T = T_, WI = WI_, WJ = WJ_, NW = WI * WJ, THREADS = 64 * NW;
  static constexpr int WTM = T / WI, WTN = T / WJ, FM = WTM / 32, FN = WTN / 32;
  static constexpr int OPER = T * 128, STAGE = 2 * OPER, LDS = 2 * STAGE;   // bytes
  static constexpr int CH = T / 8 / NW;                                       // 1 KB loads per wave, stage and operand
  static_assert(NW * WTM * WTN * 2 <= LDS, "the waves' tiles are staged in LDS");
};

// ACROSS: the accumulator of lane l holds C[l % 32][4 consecutive columns], otherwise C[4 consecutive rows][l % 32]
template <class TL, int PARTS, bool TRB, bool ACROSS>
OD_DEV void ns_product(f32x16 (&acc)[TL::FM][TL::FN], const NsOperand& A, const NsOperand& B, int kdim, char* lds) {
  constexpr int T = TL::T, CH = TL::CH;
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
      const int k = chunk * (64 / SLOTS) + lane / SLOTS, cg = (lane % SLOTS) ^ ((k & 3) << 2);
      vb[j] = (uint32_t)k * (uint32_t)(B.ld * 2) + min(cg * 8, B.rows - 8) * 2;
    } else {
      vb[j] = (uint32_t)min(row, B.rows - 1) * (uint32_t)(B.ld * 2) + kg * 16;
    }
  }
  const int ks = kdim / kNsStep, steps = ks * (PARTS == 2 ? 3 : 1);
  const int64_t bstep = TRB ? (int64_t)kNsStep * B.ld : kNsStep;
  auto issue = [&](int step) {
    const int seg = PARTS == 2 ? step / ks : 0, kk = PARTS == 2 ? step - seg * ks : step;
    const uint16_t* a = A.p + (seg == 2 ? A.plane : 0) + (int64_t)kk * kNsStep;
    const uint16_t* b = B.p + (seg == 1 ? B.plane : 0) + kk * bstep;
    const uint32_t at = lds0 + (step & 1) * TL::STAGE + wave * CH * 1024;
#pragma unroll
    for (int j = 0; j < CH; ++j) dma16_at(va[j], a, at + j * 1024);
#pragma unroll
    for (int j = 0; j < CH; ++j) dma16_at(vb[j], b, at + TL::OPER + j * 1024);
  };
#pragma unroll
  for (int i = 0; i < TL::FM; ++i)
#pragma unroll
    for (int j = 0; j < TL::FN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

  u32x4 fa[2][TL::FM], fb[2][TL::FN];
  auto fetch = [&](int step, int sub, int set) {
    const char* base = lds + (step & 1) * TL::STAGE;
    const int kg = 2 * sub + (lane >> 5);
#pragma unroll
    for (int i = 0; i < TL::FM; ++i) {
      const int row = wi * TL::WTM + 32 * i + (lane & 31);
      fa[set][i] = *reinterpret_cast<const u32x4*>(base + row * 128 + ((kg ^ swz64(row)) << 4));
    }
#pragma unroll
    for (int j = 0; j < TL::FN; ++j) {
      if constexpr (TRB) {
        const int k = sub * 16 + (lane >> 5) * 8 + ((lane & 15) >> 2);
        const int col = wj * TL::WTN + 32 * j + ((lane >> 4) & 1) * 16 + 4 * (lane & 3);
        const int at = k * (2 * T) + (((col >> 3) ^ ((k & 3) << 2)) << 4) + (col & 7) * 2;
        typedef __attribute__((address_space(3))) s16x4* lptr;
        const char* p = base + TL::OPER + at;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(p));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(p + 4 * (2 * T)));
        const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
        fb[set][j] = u32x4{l2[0], l2[1], h2[0], h2[1]};
      } else {
        const int row = wj * TL::WTN + 32 * j + (lane & 31);
        fb[set][j] = *reinterpret_cast<const u32x4*>(base + TL::OPER + row * 128 + ((kg ^ swz64(row)) << 4));
      }
    }
  };
  auto products = [&](int set) {
#pragma unroll
    for (int i = 0; i < TL::FM; ++i)
#pragma unroll
      for (int j = 0; j < TL::FN; ++j)
        acc[i][j] = ACROSS ? mfma_32x32x16<true>(fb[set][j], fa[set][i], acc[i][j])
                           : mfma_32x32x16<true>(fa[set][i], fb[set][j], acc[i][j]);
  };

  // Stage i + 1 is in flight during step i.  The last quarter of a step is multiplied from registers after the barrier
  // that frees its stage, so the first operands of the next step arrive behind products, not in front of them.
  issue(0);
  if (steps > 1) {
    issue(1);
    __builtin_amdgcn_s_waitcnt(vmcnt_only(2 * CH));
  } else {
    __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
  }
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  fetch(0, 0, 0);
  for (int i = 0; i < steps; ++i) {
    fetch(i, 1, 1);
    products(0);
    fetch(i, 2, 0);
    products(1);
    fetch(i, 3, 1);
    products(0);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (i + 2 < steps) issue(i + 2);
    if (i + 1 < steps) fetch(i + 1, 0, 0);
    products(1);
  }
}

// Writes a wave's tile of fp16 words (value * scale) row by row through its own part of LDS, 16 bytes a lane, and with
// `mirror` the transpose too.  `value(row, col, v)`: the value whose accumulator entry is v, row and column in the
// wave's tile.  Rows up to `rows` and columns up to `cols` of the matrix are written, from `crows` / `ccols` on as zero.
template <class TL, int PARTS, class V>
OD_DEV void ns_store(char* lds, V&& value, uint16_t* out, int64_t plane, int ld, int row0, int col0, int rows, int cols,
                     int valid_cols, bool mirror) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int ROWB = TL::WTN * 2, SL = ROWB / 16;       // bytes and 16-byte slots of a staged row
  static_assert(SL == 8, "a staged row is 128 bytes");
  char* mine = lds + wave * (TL::WTM * ROWB);
  // The words of all parts from one evaluation: evaluated once more for the second part, a value might be contracted
  // differently, round to another first word near a tie and leave a remainder of that one.
  u32x2 words[PARTS][TL::FM][TL::FN][4];
#pragma unroll
  for (int i = 0; i < TL::FM; ++i)
#pragma unroll
    for (int j = 0; j < TL::FN; ++j)
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4) {
        float x[4];
        value(i, j, v4, 32 * i + (lane & 31), 32 * j + 8 * v4 + 4 * (lane >> 5), x);
        uint32_t a[PARTS], b[PARTS];
        split2<PARTS>(x[0], x[1], a);
        split2<PARTS>(x[2], x[3], b);
#pragma unroll
        for (int part = 0; part < PARTS; ++part) words[part][i][j][v4] = u32x2{a[part], b[part]};
      }
#pragma unroll
  for (int part = 0; part < PARTS; ++part) {
#pragma unroll
    for (int i = 0; i < TL::FM; ++i)
#pragma unroll
      for (int j = 0; j < TL::FN; ++j)
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4) {
          const int r = 32 * i + (lane & 31), c = 32 * j + 8 * v4 + 4 * (lane >> 5);
          *reinterpret_cast<u32x2*>(mine + r * ROWB + (((c >> 3) ^ swz64(r)) << 4) + (c & 7) * 2) = words[part][i][j][v4];
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    uint16_t* o = out + part * plane;
#pragma unroll
    for (int it = 0; it < TL::WTM / 8; ++it) {
      const int r = it * 8 + (lane >> 3), slot = lane & 7;
      u32x4 w = *reinterpret_cast<const u32x4*>(mine + r * ROWB + ((slot ^ swz64(r)) << 4));
      const int row = row0 + r, col = col0 + 8 * slot;
      if (col + 8 > valid_cols) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t keep = (col + 2 * k < valid_cols ? 0xffffu : 0u) | (col + 2 * k + 1 < valid_cols ? 0xffff0000u : 0u);
          w[k] &= keep;
        }
      }
      if (row < rows && col < cols) *reinterpret_cast<u32x4*>(o + (int64_t)row * ld + col) = w;
    }
    if (mirror) {
      // lane l receives rows 8 (l / 16) .. + 7 of column l % 16 of each block of 32 rows and 16 columns
      typedef __attribute__((address_space(3))) s16x4* lptr;
#pragma unroll
      for (int rb = 0; rb < TL::WTM / 32; ++rb)
#pragma unroll
        for (int cb = 0; cb < TL::WTN / 16; ++cb) {
          const int c = cb * 16 + 4 * (lane & 3);
          s16x4 h[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int r = rb * 32 + (lane >> 4) * 8 + 4 * k + ((lane & 15) >> 2);
            h[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr)(mine + r * ROWB + (((c >> 3) ^ swz64(r)) << 4) + (c & 7) * 2));
          }
          const u32x2 l2 = __builtin_bit_cast(u32x2, h[0]), h2 = __builtin_bit_cast(u32x2, h[1]);
          u32x4 w{l2[0], l2[1], h2[0], h2[1]};
          const int mrow = col0 + cb * 16 + (lane & 15), mcol = row0 + rb * 32 + (lane >> 4) * 8;
          if (mcol + 8 > valid_cols) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t keep = (mcol + 2 * k < valid_cols ? 0xffffu : 0u) | (mcol + 2 * k + 1 < valid_cols ? 0xffff0000u : 0u);
              w[k] &= keep;
            }
          }
          if (mrow < rows && mcol < cols) *reinterpret_cast<u32x4*>(o + (int64_t)mrow * ld + mcol) = w;
        }
    }
    if (part + 1 < PARTS) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
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

struct NsPoly {
  float ca, cb, cc;       // of I, S and S S, with the scales of the stored words
};

// S = Y Y^T (POLY = false) or P = a I + b S + c S S (POLY = true)
template <class TL, int PARTS, bool POLY>
__global__ __launch_bounds__(TL::THREADS, 1) void k_ns_sym(NsArgs args, int src, NsPoly k) {
  extern __shared__ __align__(16) char lds[];
  constexpr int T = TL::T;
  const int bid = xcd_contiguous(blockIdx.x, args.total);
  const NsClass c = args.c[ns_class(args, bid)];
  const int n = (c.p + T - 1) / T, per = n * (n + 1) / 2;
  const int z = (bid - c.first) / per;
  int ti, tj;
  upper_tile((bid - c.first) - z * per, n, &ti, &tj);
  const int pp = up64(c.p), qq = up64(c.q);
  const int64_t yplane = (int64_t)pp * c.lq, splane = (int64_t)c.p * c.lp;
  uint16_t* slice = c.base + z * c.stride;
  uint16_t* S = slice + 2 * PARTS * yplane;
  uint16_t* P = S + PARTS * splane;
  const uint16_t* in = POLY ? S : slice + src * PARTS * yplane;
  const int64_t plane = POLY ? splane : yplane;
  const int ld = POLY ? c.lp : c.lq;
  const NsOperand A{in + (int64_t)ti * T * ld, plane, ld, c.p - ti * T}, B{in + (int64_t)tj * T * ld, plane, ld, c.p - tj * T};
  f32x16 acc[TL::FM][TL::FN];
  ns_product<TL, PARTS, false, true>(acc, A, B, POLY ? pp : qq, lds);
  __syncthreads();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row0 = ti * T + wave / TL::WJ * TL::WTM, col0 = tj * T + wave % TL::WJ * TL::WTN;
  ns_store<TL, PARTS>(lds, [&](int i, int j, int v4, int r, int cl, float* x) {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    const int row = row0 + r, col = col0 + cl;
    if constexpr (POLY) {
      if (row < c.p && col < pp) {
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
          const u32x2 w = *reinterpret_cast<const u32x2*>(S + part * splane + (int64_t)row * c.lp + col);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t pair = w[e];          // a bit cast of a vector's element itself would take its first one
            const f16x2 h = __builtin_bit_cast(f16x2, pair);
            s[2 * e] += (float)h[0];
            s[2 * e + 1] += (float)h[1];
          }
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = k.cc * acc[i][j][4 * v4 + e];
      if constexpr (POLY) x[e] += k.cb * s[e] + (row == col + e ? k.ca : 0.f);
    }
  }, POLY ? P : S, splane, c.lp, row0, col0, c.p, pp, c.p, ti != tj);
}

// Y' = P Y
template <class TL, int PARTS>
__global__ __launch_bounds__(TL::THREADS, 1) void k_ns_apply(NsArgs args, int src, float scale) {
  extern __shared__ __align__(16) char lds[];
  constexpr int T = TL::T;
  const int bid = xcd_contiguous(blockIdx.x, args.total);
  const NsClass c = args.c[ns_class(args, bid)];
  const int ni = (c.p + T - 1) / T, nj = (c.q + T - 1) / T;
  const int z = (bid - c.first) / (ni * nj), tl = (bid - c.first) - z * (ni * nj);
  const int ti = tl % ni, tj = tl / ni;
  const int pp = up64(c.p), qq = up64(c.q);
  const int64_t yplane = (int64_t)pp * c.lq, splane = (int64_t)c.p * c.lp;
  uint16_t* slice = c.base + z * c.stride;
  const uint16_t* P = slice + 2 * PARTS * yplane + PARTS * splane;
  const uint16_t* Y = slice + src * PARTS * yplane;
  uint16_t* out = slice + (1 - src) * PARTS * yplane;
  const NsOperand A{P + (int64_t)ti * T * c.lp, splane, c.lp, c.p - ti * T}, B{Y + tj * T, yplane, c.lq, qq - tj * T};
  f32x16 acc[TL::FM][TL::FN];
  ns_product<TL, PARTS, true, true>(acc, A, B, pp, lds);
  __syncthreads();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row0 = ti * T + wave / TL::WJ * TL::WTM, col0 = tj * T + wave % TL::WJ * TL::WTN;
  ns_store<TL, PARTS>(lds, [&](int i, int j, int v4, int, int, float* x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = scale * acc[i][j][4 * v4 + e];
  }, out, yplane, c.lq, row0, col0, c.p, qq, c.q, false);
}

// O = P Y into the caller's matrix, or its update
template <class TL, int PARTS, bool XBF, bool TALL>
__global__ __launch_bounds__(TL::THREADS, 1) void k_ns_final(NsArgs args, MuonTables t, int src, float scale, int update, float keep, float lr) {
  extern __shared__ __align__(16) char lds[];
  constexpr int T = TL::T;
  const int bid = xcd_contiguous(blockIdx.x, args.total);
  const NsClass c = args.c[ns_class(args, bid)];
  const int ni = (c.p + T - 1) / T, nj = (c.q + T - 1) / T;
  const int z = (bid - c.first) / (ni * nj), tl = (bid - c.first) - z * (ni * nj);
  const int ti = tl % ni, tj = tl / ni;
  const int pp = up64(c.p), qq = up64(c.q);
  const int64_t yplane = (int64_t)pp * c.lq, splane = (int64_t)c.p * c.lp;
  uint16_t* slice = c.base + z * c.stride;
  const uint16_t* P = slice + 2 * PARTS * yplane + PARTS * splane;
  const uint16_t* Y = slice + src * PARTS * yplane;
  const NsOperand A{P + (int64_t)ti * T * c.lp, splane, c.lp, c.p - ti * T}, B{Y + tj * T, yplane, c.lq, qq - tj * T};
  f32x16 acc[TL::FM][TL::FN];
  ns_product<TL, PARTS, true, !TALL>(acc, A, B, pp, lds);
  const MuonMat a = t.mats[c.mat0 + z];
  const MuonEntry e = t.entries[c.mat0 + z];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i0 = ti * T + wave / TL::WJ * TL::WTM, j0 = tj * T + wave % TL::WJ * TL::WTN;
  const bool vec = (reinterpret_cast<uintptr_t>(e.X) & (XBF ? 7 : 15)) == 0 && (a.ldx & 3) == 0;
  const float step = update ? lr * a.scale * scale : -scale;
  const float kx = update ? keep : 0.f;
#pragma unroll
  for (int i = 0; i < TL::FM; ++i)
#pragma unroll
    for (int j = 0; j < TL::FN; ++j)
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4) {
        const int run = 8 * v4 + 4 * (lane >> 5);
        const int row = TALL ? j0 + 32 * j + (lane & 31) : i0 + 32 * i + (lane & 31);
        const int col = TALL ? i0 + 32 * i + run : j0 + 32 * j + run;
        if (row >= a.m || col >= a.n) continue;
        const int64_t at = (int64_t)row * a.ldx + col;
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        if (vec && col + 4 <= a.n) {
          if constexpr (XBF) {
            u32x2* px = reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(e.X) + at);
            if (update) SrcBF16::unpack4(*px, x);
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = kx * x[k] - step * acc[i][j][4 * v4 + k];
            *px = u32x2{pack_bf16_rne(x[0], x[1]), pack_bf16_rne(x[2], x[3])};
          } else {
            f32x4* px = reinterpret_cast<f32x4*>(reinterpret_cast<float*>(e.X) + at);
            if (update) SrcF32::unpack4(*px, x);
            f32x4 o;
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = kx * x[k] - step * acc[i][j][4 * v4 + k];
            *px = o;
          }
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (col + k >= a.n) continue;
            if (update) x[k] = load_elem<XBF>(e.X, at + k);
            const float o = kx * x[k] - step * acc[i][j][4 * v4 + k];
            if constexpr (XBF) reinterpret_cast<uint16_t*>(e.X)[at + k] = (uint16_t)pack_bf16_rne(o, 0.f);
            else reinterpret_cast<float*>(e.X)[at + k] = o;
          }
        }
      }
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

// the classes that `take` accepts, with the workgroups that `tiles` gives per matrix
template <class Take, class Tiles>
NsArgs laid_out(const NsArgs& a, Take&& take, Tiles&& tiles) {
  NsArgs o = {};
  for (int k = 0; k < a.nclass; ++k) {
    if (!take(a.c[k])) continue;
    o.c[o.nclass] = a.c[k];
    o.c[o.nclass++].first = o.total;
    o.total += a.c[k].nb * tiles(a.c[k]);
  }
  return o;
}

int ceil_div(int a, int b) { return (a + b - 1) / b; }
bool any(const NsClass&) { return true; }

// more than 64 KB of LDS have to be asked for, once per kernel and device
template <class K>
hipError_t allow_lds(K* kernel, int bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <class TL, class K, class... A>
hipError_t go(K* kernel, const NsArgs& a, hipStream_t st, A... rest) {
  if (a.total == 0) return hipSuccess;
  if (TL::LDS > 65536) {
    const hipError_t rc = allow_lds(kernel, TL::LDS);
    if (rc != hipSuccess) return rc;
  }
  kernel<<<a.total, TL::THREADS, TL::LDS, st>>>(a, rest...);
  return hipGetLastError();
}

typedef NsTile<128, 2, 2> Small;

template <class TL>
NsArgs upper(const NsArgs& a) {
  return laid_out(a, any, [](const NsClass& c) { const int n = ceil_div(c.p, TL::T); return n * (n + 1) / 2; });
}
template <class TL>
int full(const NsClass& c) { return ceil_div(c.p, TL::T) * ceil_div(c.q, TL::T); }

template <class TL, int PARTS, bool XBF>
hipError_t final_of(const NsArgs& a, const MuonTables& t, int src, float s, bool update, float keep, float lr, hipStream_t st) {
  const hipError_t rc = go<TL>(k_ns_final<TL, PARTS, XBF, false>, laid_out(a, [](const NsClass& c) { return !c.tall; }, full<TL>), st, t, src, s, (int)update, keep, lr);
  if (rc != hipSuccess) return rc;
  return go<TL>(k_ns_final<TL, PARTS, XBF, true>, laid_out(a, [](const NsClass& c) { return c.tall != 0; }, full<TL>), st, t, src, s, (int)update, keep, lr);
}

}  // namespace

hipError_t launch_muon_scale(const NsArgs& a, const MuonTables& t, float mu, bool nesterov, bool g_bf16, int parts, double eps,
                             double scale, hipStream_t st) {
  const NsArgs o = laid_out(a, any, [](const NsClass& c) { return ceil_div(c.p, 64) * ceil_div(c.q, 64); });
  auto run = [&](auto kernel) { kernel<<<o.total, 256, 0, st>>>(o, t, mu, (int)nesterov, eps, scale); };
  if (g_bf16) parts == 2 ? run(k_muon_scale<true, 2>) : run(k_muon_scale<true, 1>);
  else parts == 2 ? run(k_muon_scale<false, 2>) : run(k_muon_scale<false, 1>);
  return hipGetLastError();
}

hipError_t launch_ns_gram(const NsArgs& a, int parts, int src, float out_scale, hipStream_t st) {
  const NsPoly k{0.f, 0.f, out_scale};
  const NsArgs o = upper<Small>(a);
  return parts == 2 ? go<Small>(k_ns_sym<Small, 2, false>, o, st, src, k) : go<Small>(k_ns_sym<Small, 1, false>, o, st, src, k);
}

hipError_t launch_ns_poly(const NsArgs& a, int parts, float ca, float cb, float cc, float s_scale, float out_scale, hipStream_t st) {
  const NsPoly k{ca * out_scale, cb * out_scale / s_scale, cc * out_scale / (s_scale * s_scale)};
  const NsArgs o = upper<Small>(a);
  return parts == 2 ? go<Small>(k_ns_sym<Small, 2, true>, o, st, 0, k) : go<Small>(k_ns_sym<Small, 1, true>, o, st, 0, k);
}

hipError_t launch_ns_apply(const NsArgs& a, int parts, int src, float out_scale, hipStream_t st) {
  const NsArgs o = laid_out(a, any, full<Small>);
  return parts == 2 ? go<Small>(k_ns_apply<Small, 2>, o, st, src, out_scale) : go<Small>(k_ns_apply<Small, 1>, o, st, src, out_scale);
}

hipError_t launch_ns_final(const NsArgs& a, const MuonTables& t, int parts, int src, float out_scale, bool update, float keep, float lr,
                           bool x_bf16, hipStream_t st) {
  if (parts == 2)
    return x_bf16 ? final_of<Small, 2, true>(a, t, src, out_scale, update, keep, lr, st) : final_of<Small, 2, false>(a, t, src, out_scale, update, keep, lr, st);
  return x_bf16 ? final_of<Small, 1, true>(a, t, src, out_scale, update, keep, lr, st) : final_of<Small, 1, false>(a, t, src, out_scale, update, keep, lr, st);
}

}  // namespace od
