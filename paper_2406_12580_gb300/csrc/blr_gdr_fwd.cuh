// Forward kernels of the gated delta rule, in chunks of C = 64 steps. With the
// chunk's cumulative log decay G, gamma_i = e^{G_i}, S the state before it:
//     A_ij = beta_i e^{G_i - G_j} k_i.k_j (j < i),  T = (I + A)^-1
//     U = T diag(beta) V - [T diag(beta gamma) K] S = U0 - W S
//     S' = gamma_C S + K^T diag(e^{G_C - G}) U
//     O = scale (diag(gamma) Q S + P U),  P_ij = e^{G_i - G_j} q_i.k_j (j <= i)
// Three kernels: `prepare` (all chunks at once: T, W, U0), `chain` (the only
// serial part: two products a chunk, U and S'), `output` (all chunks at once).
#pragma once

#include "blr_gdr_tile.cuh"

namespace blr {
namespace gdr {

// The chunk's gates: cumulative log decay and beta, zero on slots past the end. With two planes the sum
// is a pair of floats: a difference of two sums near -1000 keeps its last bits.
template <int P, typename T>
__device__ __forceinline__ void load_gates(const T* g, const T* beta, int64_t stride, int rows,
                                           float* out) {  // by one warp; `out`: kGates floats
  using Sum = typename std::conditional<(P > 1), double, float>::type;
  const int l = threadIdx.x & 31;
  const Sum x = 2 * l < rows ? fmaxf(to_float(g[2 * l * stride]), kMinDecay) : 0.0f;
  const Sum y = 2 * l + 1 < rows ? fmaxf(to_float(g[(2 * l + 1) * stride]), kMinDecay) : 0.0f;
  Sum s = x + y;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const Sum o = __shfl_up_sync(0xffffffffu, s, d);
    if (l >= d) s += o;
  }
  const Sum G[2] = {s - y, s}, last = __shfl_sync(0xffffffffu, s, 31);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int i = 2 * l + e;
    out[i] = (float)G[e];
    out[kBeta + i] = i < rows ? to_float(beta[i * stride]) : 0.0f;
    out[kUp + i] = exp_p<P>((float)G[e]);
    out[kDown + i] = exp_p<P>((float)(last - G[e]));
    if constexpr (P > 1) out[kRest + i] = (float)(G[e] - (Sum)(float)G[e]);
  }
}

constexpr int kLd = 68;  // row stride of float32 squares in shared memory: fragment reads meet all banks

// Block column J of T^-1's lower triangle from the inverses of the diagonal blocks (already in `inv`):
// T_iJ = -T_ii sum_{J <= m < i} A_im T_mJ, kept transposed so that an accumulator is the next left operand.
template <int J, int P>
__device__ __forceinline__ void inverse_column(const float* A, float* inv) {
  const int l = threadIdx.x & 31, r = l >> 2, c = 2 * (l & 3);
  float t[4][2][4];  // T_mJ^T, m = J..3: 16 x 16 as two column blocks
#pragma unroll
  for (int nb = 0; nb < 2; ++nb)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      t[J][nb][e] = inv[(16 * J + 8 * nb + c + (e & 1)) * kLd + 16 * J + r + 8 * (e >> 1)];
  auto right = [&](const float* m, int row0, int col0, uint32_t (&b)[2][kPl<P>][2]) {  // of m^T's block
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const float2 v = *reinterpret_cast<const float2*>(&m[(row0 + 8 * nb + r) * kLd + col0 + 8 * kb + c]);
        uint32_t w[kPl<P>];
        split2<P>(v.x, v.y, w);
#pragma unroll
        for (int p = 0; p < kPl<P>; ++p) b[nb][p][kb] = w[p];
      }
  };
#pragma unroll
  for (int i = J + 1; i < 4; ++i) {
    float s[2][4] = {};
#pragma unroll
    for (int m = J; m < i; ++m) {
      uint32_t a[kPl<P>][4], b[2][kPl<P>][2];
      to_a<P>(t[m][0], t[m][1], a);
      right(A, 16 * i, 16 * m, b);
      mma_p<P, P>(s[0], a, b[0]);
      mma_p<P, P>(s[1], a, b[1]);
    }
    uint32_t a[kPl<P>][4], b[2][kPl<P>][2];
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[nb][e] = -s[nb][e];
        t[i][nb][e] = 0.0f;
      }
    to_a<P>(s[0], s[1], a);
    right(inv, 16 * i, 16 * i, b);
    mma_p<P, P>(t[i][0], a, b[0]);
    mma_p<P, P>(t[i][1], a, b[1]);
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        inv[(16 * i + 8 * nb + c + (e & 1)) * kLd + 16 * J + r + 8 * (e >> 1)] = t[i][nb][e];
  }
}

template <int DK, int NI, int NM>
struct PrepareSmem {
  static constexpr int kK = Tile<DK / 8, NI>::kBytes, kV = Tile<8, NI>::kBytes;
  static constexpr int kSquare = 64 * kLd * 4;
  static constexpr int kBytes = kK + kV + 2 * kSquare + kGates * 4;
};

// T, W = T diag(beta gamma) K (stored negated), U0 = T diag(beta) V of one chunk of one head. A warp
// holds 16 rows of the chunk. The diagonal 16 x 16 blocks of T by substitution in float32, the rest by
// products of two planes at least, whatever the operands of the rest.
template <typename TI, int DK, int NI, int NM, bool TRAIN>
__global__ void __launch_bounds__(128)
prepare_kernel(const Problem P, const TI* __restrict__ k, const TI* __restrict__ v, const TI* __restrict__ g,
               const TI* __restrict__ beta) {
  extern __shared__ __align__(128) unsigned char smem[];
  using L = PrepareSmem<DK, NI, NM>;
  const Tile<DK / 8, NI> tk{smem_u32(smem)};
  const Tile<8, NI> tv{smem_u32(smem) + L::kK};
  float* A = reinterpret_cast<float*>(smem + L::kK + L::kV);
  float* inv = A + 64 * kLd;
  float* sg = inv + 64 * kLd;  // the gates
  float* sb = sg + 64;
  const Where w = locate(P);
  if (w.rows <= 0) return;
  const int tid = threadIdx.x, warp = tid >> 5, l = tid & 31;
  const int64_t row0 = w.step;
  load_rows<128>(tk, k + row0 * P.ldk + w.hk * DK, P.ldk, w.rows, tid);
  load_rows<128>(tv, v + row0 * P.ldv + (int64_t)w.h * P.Dv, P.ldv, w.rows, tid);
  cp_async_commit();
  if (warp == 0) {
    load_gates<NM>(g + row0 * P.Hv + w.h, beta + row0 * P.Hv + w.h, P.Hv, w.rows, sg);
    __syncwarp();
    float* out = P.gates + w.nc * kGates;
#pragma unroll
    for (int i = 0; i < kGateFloats<NM>; i += 64)
      *reinterpret_cast<float2*>(out + i + 2 * l) = *reinterpret_cast<float2*>(sg + i + 2 * l);
  }
  cp_async_wait<0>();
  __syncthreads();
  const int r0 = 16 * warp + (l >> 2), c0 = 2 * (l & 3);
  {  // A
    float acc[8][4] = {};
#pragma unroll
    for (int kk = 0; kk < DK / 16; ++kk) {
      uint32_t a[kPl<NI>][4];
      tk.a(2 * warp, 2 * kk, a);
#pragma unroll
      for (int nn = 0; nn < 4; ++nn) {
        if (nn <= warp) {
          uint32_t b[2][kPl<NI>][2];
          tk.b_t(2 * nn, 2 * kk, b);
          mma_p<NI, NI>(acc[2 * nn], a, b[0]);
          mma_p<NI, NI>(acc[2 * nn + 1], a, b[1]);
        }
      }
    }
#pragma unroll
    for (int nb = 0; nb < 8; ++nb)
      if (nb < 2 * warp + 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = r0 + 8 * (e >> 1), j = 8 * nb + c0 + (e & 1);
          A[i * kLd + j] = j < i ? sb[i] * decay_between<NM>(sg, i, j) * acc[nb][e] : 0.0f;
        }
      }
  }
  __syncwarp();
  {  // the diagonal block's inverse: lane c solves (I + A_ww) x = e_c
    const int c = l & 15;
    const float* Aw = A + 16 * warp * kLd + 16 * warp;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float s = i == c ? 1.0f : 0.0f;
#pragma unroll
      for (int m = 0; m < 16; ++m)
        if (m < i) s = fmaf(-Aw[i * kLd + m], x[m], s);
      x[i] = s;
    }
    if (l < 16) {
#pragma unroll
      for (int i = 0; i < 16; ++i) inv[(16 * warp + i) * kLd + 16 * warp + c] = x[i];
    }
  }
  __syncthreads();
  constexpr int kInv = NM == 3 ? 3 : 2;
  if (warp == 0) inverse_column<0, kInv>(A, inv);
  else if (warp == 1) inverse_column<1, kInv>(A, inv);
  else if (warp == 2) inverse_column<2, kInv>(A, inv);
  __syncthreads();
  // rows of T, scaled by column, as left operands
  const auto rows_of_t = [&](int kk, const float* scale, uint32_t (&a)[kPl<NM>][4]) {
    float x[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int j = 16 * kk + 8 * h + c0;
      const float s0 = scale == nullptr ? 1.0f : scale[j], s1 = scale == nullptr ? 1.0f : scale[j + 1];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float2 t = *reinterpret_cast<const float2*>(&inv[(r0 + 8 * e) * kLd + j]);
        x[h][2 * e] = t.x * s0;
        x[h][2 * e + 1] = t.y * s1;
      }
    }
    to_a<NM>(x[0], x[1], a);
  };
  if constexpr (TRAIN) {
    char* t = P.T + w.nc * Tile<8, NM>::kBytes;
    for (int nb = 0; nb < 2 * warp + 2; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float2 x = *reinterpret_cast<const float2*>(&inv[(r0 + 8 * e) * kLd + 8 * nb + c0]);
        store_block<8, NM>(t, 2 * warp + e, nb, x.x, x.y);
      }
  }
  // U0, 64 columns of V at a time
  const int dvb = P.Dv / 64;
  for (int part = 0; part < dvb; ++part) {
    if (part > 0) {
      __syncthreads();
      load_rows<128>(tv, v + row0 * P.ldv + (int64_t)w.h * P.Dv + 64 * part, P.ldv, w.rows, tid);
      cp_async_commit();
      cp_async_wait<0>();
      __syncthreads();
    }
    float acc[8][4] = {};
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
      if (kk <= warp) {
        uint32_t a[kPl<NM>][4];
        rows_of_t(kk, sb, a);
#pragma unroll
        for (int nn = 0; nn < 4; ++nn) {
          uint32_t b[2][kPl<NI>][2];
          tv.b(2 * nn, 2 * kk, b);
          mma_p<NM, NI>(acc[2 * nn], a, b[0]);
          mma_p<NM, NI>(acc[2 * nn + 1], a, b[1]);
        }
      }
    char* u = P.U + (w.nc * dvb + part) * Tile<8, NM>::kBytes;
#pragma unroll
    for (int nb = 0; nb < 8; ++nb) {
      store_block<8, NM>(u, 2 * warp, nb, acc[nb][0], acc[nb][1]);
      store_block<8, NM>(u, 2 * warp + 1, nb, acc[nb][2], acc[nb][3]);
    }
  }
  // -W: the column scale becomes -beta gamma
  __syncthreads();
  if (tid < 64) sb[tid] *= -sg[kUp + tid];
  __syncthreads();
  char* wt = P.W + w.nc * Tile<DK / 8, NM>::kBytes;
#pragma unroll
  for (int half = 0; half < DK / 64; ++half) {
    float acc[8][4] = {};
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
      if (kk <= warp) {
        uint32_t a[kPl<NM>][4];
        rows_of_t(kk, sb, a);
#pragma unroll
        for (int nn = 0; nn < 4; ++nn) {
          uint32_t b[2][kPl<NI>][2];
          tk.b(8 * half + 2 * nn, 2 * kk, b);
          mma_p<NM, NI>(acc[2 * nn], a, b[0]);
          mma_p<NM, NI>(acc[2 * nn + 1], a, b[1]);
        }
      }
#pragma unroll
    for (int nb = 0; nb < 8; ++nb) {
      store_block<DK / 8, NM>(wt, 2 * warp, 8 * half + nb, acc[nb][0], acc[nb][1]);
      store_block<DK / 8, NM>(wt, 2 * warp + 1, 8 * half + nb, acc[nb][2], acc[nb][3]);
    }
  }
}

template <int DK, int NI, int NM, int WARPS>
struct ChainSmem {
  static constexpr int kW = Tile<DK / 8, NM>::kBytes, kK = Tile<DK / 8, NI>::kBytes, kU = Tile<2 * WARPS, NM>::kBytes;
  static constexpr int kStage = kW + kK + kU + kGates * 4;
  static constexpr int kStages = WARPS == 2 && 3 * kStage <= 227 * 1024 ? 3 : 2;
  static constexpr int kBytes = kStages * kStage;
};

// The states from chunk to chunk. A block takes 16 WARPS columns of a head's state, a warp 16 of them, as
// S^T (16 x Dk) in accumulators: U^T = U0^T + S^T (-W)^T and S'^T = gamma_C S^T + (U^T diag(e^{G_C - G})) K
// take their left operands from registers, so the warps of a head never exchange anything; the block
// shares only the tiles that it streams. Two more warps only load, kStages - 1 chunks ahead: one barrier a
// chunk says both that a stage has arrived and that the one before it may be filled again.
template <typename TI, int DK, int NI, int NM, int WARPS>
__global__ void __launch_bounds__(32 * (WARPS + kLoadWarps), WARPS == 4 && NM < 3 ? 2 : 1)
chain_kernel(const Problem P, const TI* __restrict__ k, const float* __restrict__ s0,
             float* __restrict__ s_last) {
  extern __shared__ __align__(128) unsigned char smem[];
  using L = ChainSmem<DK, NI, NM, WARPS>;
  const int parts = P.Dv / (16 * WARPS), dvb = P.Dv / 64;
  const uint32_t bh = blockIdx.x / parts;
  const int part = blockIdx.x - bh * parts;
  const int warp = threadIdx.x >> 5, l = threadIdx.x & 31;
  const Where w0 = locate(P, bh, 0);
  const int chunks = (int)((w0.len + kC - 1) / kC);
  const int block = part * WARPS / 4, c8 = 2 * ((part * WARPS) & 3);  // this part's 64 columns, and where in them
  if (warp >= WARPS) {  // loads
    const int tid = threadIdx.x - 32 * WARPS;
    const auto load = [&](int c) {
      if (c < chunks) {
        const uint32_t st = smem_u32(smem) + (uint32_t)(c % L::kStages) * L::kStage;
        const int64_t nc = w0.nc + c, left = w0.len - (int64_t)c * kC;
        copy_ws<L::kW, 32 * kLoadWarps>(st, P.W + nc * L::kW, tid);
        load_rows<32 * kLoadWarps>(Tile<DK / 8, NI>{st + L::kW}, k + (w0.step + (int64_t)c * kC) * P.ldk + w0.hk * DK,
                                   P.ldk, (int)(left < kC ? left : kC), tid);
        copy_columns<32 * kLoadWarps>(Tile<2 * WARPS, NM>{st + L::kW + L::kK}, P.U + (nc * dvb + block) * Tile<8, NM>::kBytes, c8, tid);
        copy_ws<1024, 32 * kLoadWarps>(st + L::kW + L::kK + L::kU, P.gates + nc * kGates, tid);
      }
      cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < L::kStages - 1; ++i) load(i);
    for (int c = 0; c < chunks; ++c) {
      cp_async_wait<L::kStages - 2>();
      __syncthreads();
      load(c + L::kStages - 1);
    }
    return;
  }
  const int col = 16 * (part * WARPS + warp) + (l >> 2), row = 2 * (l & 3);  // of S (row + 8 nb, col (+ 8))
  float S[DK / 8][4];
#pragma unroll
  for (int nb = 0; nb < DK / 8; ++nb)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      S[nb][e] = s0 == nullptr ? 0.0f : s0[((int64_t)bh * DK + 8 * nb + row + (e & 1)) * P.Dv + col + 8 * (e >> 1)];
  for (int c = 0; c < chunks; ++c) {
    __syncthreads();
    const int s = c % L::kStages;
    const uint32_t st = smem_u32(smem) + s * L::kStage;
    const Tile<DK / 8, NM> tw{st};
    const Tile<DK / 8, NI> tk{st + L::kW};
    const Tile<2 * WARPS, NM> tu{st + L::kW + L::kK};
    const float* G = reinterpret_cast<const float*>(smem + s * L::kStage + L::kW + L::kK + L::kU);
    const int64_t tile = (w0.nc + c) * dvb + block;
    float u[8][4];
#pragma unroll
    for (int nb = 0; nb < 8; nb += 2) {  // U0^T: blocks (tokens 8 nb, columns 16 warp), transposed
      uint32_t f[2][kPl<NM>][2];
      const int i = l >> 3;
#pragma unroll
      for (int p = 0; p < kPl<NM>; ++p)
        ldsm_t(tu.at(p, nb + (i >> 1), 2 * warp + (i & 1)) + (l & 7) * 16, f[0][p][0], f[0][p][1], f[1][p][0],
               f[1][p][1]);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          uint32_t x[kPl<NM>];
#pragma unroll
          for (int p = 0; p < kPl<NM>; ++p) x[p] = f[h][p][e];
          const float2 v = join2<NM>(x);
          u[nb + h][2 * e] = v.x;
          u[nb + h][2 * e + 1] = v.y;
        }
    }
    // the state before the chunk goes out as it becomes an operand: blocks (columns 16 warp.., rows 16 kk..)
    char* so = P.S + tile * Tile<DK / 8, NM>::kBytes + (c8 + 2 * warp) * (DK / 8) * 128 + l * 4;
    pipelined<DK / 16, 4, NM>(
        [&](int kk, auto& b) {
#pragma unroll
          for (int nn = 0; nn < 4; ++nn) tw.b_t(2 * nn, 2 * kk, b[nn]);
        },
        [&](int kk, auto& b) {
          uint32_t a[kPl<NM>][4];
          to_a<NM>(S[2 * kk], S[2 * kk + 1], a);
#pragma unroll
          for (int p = 0; p < kPl<NM>; ++p)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              *reinterpret_cast<uint32_t*>(so + p * Tile<DK / 8, NM>::kPlane +
                                           ((e & 1) * (DK / 8) + 2 * kk + (e >> 1)) * 128) = a[p][e];
#pragma unroll
          for (int nn = 0; nn < 4; ++nn) {
            mma_p<NM, NM>(u[2 * nn], a, b[nn][0]);
            mma_p<NM, NM>(u[2 * nn + 1], a, b[nn][1]);
          }
        });
    const float decay = G[kUp + 63];
#pragma unroll
    for (int nb = 0; nb < DK / 8; ++nb)
#pragma unroll
      for (int e = 0; e < 4; ++e) S[nb][e] *= decay;
    char* uo = P.U + tile * Tile<8, NM>::kBytes;
    uint32_t a[kPl<NM>][4];
    pipelined<4 * (DK / 64), 4, NI>(
        [&](int s, auto& b) {
          const int kk = s / (DK / 64), n0 = 8 * (s % (DK / 64));
#pragma unroll
          for (int nn = 0; nn < 4; ++nn) tk.b(n0 + 2 * nn, 2 * kk, b[nn]);
        },
        [&](int s, auto& b) {
          const int kk = s / (DK / 64), n0 = 8 * (s % (DK / 64));
          if (n0 == 0) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float(&x)[4] = u[2 * kk + h];
              store_block_t<8, NM>(uo, 2 * kk + h, c8 + 2 * warp, x[0], x[1]);
              store_block_t<8, NM>(uo, 2 * kk + h, c8 + 2 * warp + 1, x[2], x[3]);
              const float2 down = *reinterpret_cast<const float2*>(&G[kDown + 16 * kk + 8 * h + row]);
              x[0] *= down.x;
              x[1] *= down.y;
              x[2] *= down.x;
              x[3] *= down.y;
            }
            to_a<NM>(u[2 * kk], u[2 * kk + 1], a);
          }
#pragma unroll
          for (int nn = 0; nn < 4; ++nn) {
            mma_p<NM, NI>(S[n0 + 2 * nn], a, b[nn][0]);
            mma_p<NM, NI>(S[n0 + 2 * nn + 1], a, b[nn][1]);
          }
        });
  }
  if (s_last != nullptr) {
#pragma unroll
    for (int nb = 0; nb < DK / 8; ++nb)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s_last[((int64_t)bh * DK + 8 * nb + row + (e & 1)) * P.Dv + col + 8 * (e >> 1)] = S[nb][e];
  }
}

template <int DK, int NI, int NM>
struct OutputSmem {
  static constexpr int kQ = Tile<DK / 8, NI>::kBytes, kU = Tile<8, NM>::kBytes, kS = Tile<DK / 8, NM>::kBytes;
  static constexpr int kBytes = 2 * kQ + kU + kS + kGates * 4;
};

// O = scale (diag(gamma) Q S + P U) of one chunk of one head; zero on the row's padding.
template <typename TI, int DK, int NI, int NM>
__global__ void __launch_bounds__(128)
output_kernel(const Problem P, const TI* __restrict__ q, const TI* __restrict__ k, TI* __restrict__ o) {
  extern __shared__ __align__(128) unsigned char smem[];
  using L = OutputSmem<DK, NI, NM>;
  const Where w = locate(P);
  const int tid = threadIdx.x, warp = tid >> 5, l = tid & 31;
  if (w.rows < kC && w.len < P.L) {
    for (int i = tid; i < kC * (P.Dv / 2); i += 128) {
      const int64_t t = padding_step(P, w, i / (P.Dv / 2));
      if (t >= 0) store_pair(o + ((w.b * P.L + t) * P.Hv + w.h) * P.Dv + 2 * (i % (P.Dv / 2)), 0.0f, 0.0f);
    }
  }
  if (w.rows <= 0) return;
  const uint32_t base = smem_u32(smem);
  const Tile<DK / 8, NI> tq{base}, tk{base + L::kQ};
  const Tile<8, NM> tu{base + 2 * L::kQ};
  const Tile<DK / 8, NM> ts{base + 2 * L::kQ + L::kU};
  float* G = reinterpret_cast<float*>(smem + 2 * L::kQ + L::kU + L::kS);
  const int64_t row0 = w.step;
  const int dvb = P.Dv / 64;
  load_rows<128>(tq, q + row0 * P.ldq + w.hk * DK, P.ldq, w.rows, tid);
  load_rows<128>(tk, k + row0 * P.ldk + w.hk * DK, P.ldk, w.rows, tid);
  copy_ws<4 * kGateFloats<NM>, 128>(smem_u32(G), P.gates + w.nc * kGates, tid);
  cp_async_commit();
  const auto load = [&](int part) {
    copy_ws<L::kU, 128>(tu.base, P.U + (w.nc * dvb + part) * L::kU, tid);
    copy_ws<L::kS, 128>(ts.base, P.S + (w.nc * dvb + part) * L::kS, tid);
    cp_async_commit();
  };
  load(0);
  cp_async_wait<1>();
  __syncthreads();
  const int r = l >> 2, c0 = 2 * (l & 3), r0 = 16 * warp + r;
  uint32_t p[4][kPl<NM>][4];  // P, as left operands
  {
    float acc[8][4] = {};
#pragma unroll
    for (int kk = 0; kk < DK / 16; ++kk) {
      uint32_t a[kPl<NI>][4];
      tq.a(2 * warp, 2 * kk, a);
#pragma unroll
      for (int nn = 0; nn < 4; ++nn)
        if (nn <= warp) {
          uint32_t b[2][kPl<NI>][2];
          tk.b_t(2 * nn, 2 * kk, b);
          mma_p<NI, NI>(acc[2 * nn], a, b[0]);
          mma_p<NI, NI>(acc[2 * nn + 1], a, b[1]);
        }
    }
#pragma unroll
    for (int nb = 0; nb < 8; ++nb)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = r0 + 8 * (e >> 1), j = 8 * nb + c0 + (e & 1);
        acc[nb][e] = j <= i ? acc[nb][e] * decay_between<NM>(G, i, j) : 0.0f;
      }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) to_a<NM>(acc[2 * kk], acc[2 * kk + 1], p[kk]);
  }
  const float up0 = G[kUp + r0], up1 = G[kUp + r0 + 8];
  for (int part = 0; part < dvb; ++part) {
    if (part > 0) {
      __syncthreads();
      load(part);
    }
    cp_async_wait<0>();
    __syncthreads();
    float acc[8][4] = {};
#pragma unroll
    for (int kk = 0; kk < DK / 16; ++kk) {
      uint32_t a[kPl<NI>][4];
      tq.a(2 * warp, 2 * kk, a);
#pragma unroll
      for (int nn = 0; nn < 4; ++nn) {
        uint32_t b[2][kPl<NM>][2];
        ts.b_t(2 * nn, 2 * kk, b);
        mma_p<NI, NM>(acc[2 * nn], a, b[0]);
        mma_p<NI, NM>(acc[2 * nn + 1], a, b[1]);
      }
    }
#pragma unroll
    for (int nb = 0; nb < 8; ++nb) {
      acc[nb][0] *= up0;
      acc[nb][1] *= up0;
      acc[nb][2] *= up1;
      acc[nb][3] *= up1;
    }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
      if (kk <= warp) {
#pragma unroll
        for (int nn = 0; nn < 4; ++nn) {
          uint32_t b[2][kPl<NM>][2];
          tu.b(2 * nn, 2 * kk, b);
          mma_p<NM, NM>(acc[2 * nn], p[kk], b[0]);
          mma_p<NM, NM>(acc[2 * nn + 1], p[kk], b[1]);
        }
      }
    TI* out = o + ((row0 + r0) * P.Hv + w.h) * P.Dv + 64 * part + c0;
#pragma unroll
    for (int nb = 0; nb < 8; ++nb) {
      if (r0 < w.rows) store_pair(out + 8 * nb, P.scale * acc[nb][0], P.scale * acc[nb][1]);
      if (r0 + 8 < w.rows)
        store_pair(out + 8 * P.Hv * (int64_t)P.Dv + 8 * nb, P.scale * acc[nb][2], P.scale * acc[nb][3]);
    }
  }
}

}  // namespace gdr
}  // namespace blr
