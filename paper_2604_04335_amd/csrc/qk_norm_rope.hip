// The rotation table of token positions, and the norm and rotation of queries and keys for each head.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qk_norm_rope.h"
#include "store_through.h"

namespace dit {

typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

// ---------------------------------------------------------------------------------------------
// table[r, j] = magnitude * (cos, sin)(2 pi * position * turns_j).
//
// Angles of far positions have no bits left behind the point in 32 bits, so turns are counted in double: the product with the
// position as a double and its error (fma), whole turns taken off exactly, then the nearest quarter turn.  What is left, an
// eighth of a turn at most, is an fp32 angle with its relative precision, whose sine and cosine are short Taylor sums (the
// first terms left out are under 2e-9); the quarter selects and signs them.
// A thread keeps one pair and goes down the rows.
// ---------------------------------------------------------------------------------------------
constexpr int kTableRows = 8;  // rows per thread

__global__ void __launch_bounds__(256) rope_table_kernel(RopeTableParams p) {
  const uint32_t n_pairs = (uint32_t)p.n_pairs, per = 256 / n_pairs;  // rows side by side in a workgroup
  const uint32_t sub = threadIdx.x / n_pairs, pair = threadIdx.x - sub * n_pairs;
  if (sub >= per) return;
  const double hi = p.turns_hi[pair], lo = p.turns_lo[pair];
  const int axis = p.axis[pair];
  const int64_t r0 = (int64_t)blockIdx.x * (per * kTableRows) + sub;
#pragma unroll
  for (int i = 0; i < kTableRows; ++i) {
    const int64_t r = r0 + (int64_t)i * per;
    if (r >= p.n_rows) return;
    const double pos = (double)p.positions[r * p.n_axes + axis];
    const double t = pos * hi, err = __builtin_fma(pos, hi, -t) + pos * lo;
    const double frac = (t - __builtin_rint(t)) + err;
    const double quarter = __builtin_rint(4.0 * frac);
    const float x = (float)((frac - 0.25 * quarter) * 6.283185307179586476925), x2 = x * x;
    const float s = x + x * x2 * (-1.f / 6 + x2 * (1.f / 120 + x2 * (-1.f / 5040 + x2 * (1.f / 362880))));
    const float c = 1.f - 0.5f * x2 + x2 * x2 * (1.f / 24 + x2 * (-1.f / 720 + x2 * (1.f / 40320 - x2 * (1.f / 3628800))));
    const int q = (int)quarter & 3;
    const float cq = q & 1 ? s : c, sq = q & 1 ? c : s;
    const f32x2 cs = {p.magnitude * (q == 1 || q == 2 ? -cq : cq), p.magnitude * (q >= 2 ? -sq : sq)};
    *reinterpret_cast<f32x2*>(p.table + (r * n_pairs + pair) * 2) = cs;
  }
}

hipError_t rope_table_launch(const RopeTableParams& p, hipStream_t stream) {
  if (p.n_rows == 0) return hipSuccess;
  const int64_t rows = (256 / p.n_pairs) * kTableRows, blocks = (p.n_rows + rows - 1) / rows;
  if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, p);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Norm and rotation.  D / 8 lanes share a (row, head), eight elements each, in registers from the load to the store: every
// byte is read and written once, rounded once, and a head may be replaced in place.  HBM bound, 4 D bytes a head and row.
//
// Pairs lie in one lane: with the interleaved layout a lane holds elements 8t .. 8t+7; with halves the first rot/8 lanes
// hold 4t .. 4t+3 and rot/2 + 4t .. +3.  Either way the lane's pairs are 4t .. 4t+3 of the table.  Table, weights and biases
// are loaded once for kHeads heads of the row.
// ---------------------------------------------------------------------------------------------
constexpr int kHeads = 4;

// Sum over the aligned groups of N lanes (N = 8 or 16), in all of them.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
template <int N>
__device__ __forceinline__ float group_sum(float x) {
  x = dpp_add<0xB1>(x);   // quad_perm: lane ^ 1
  x = dpp_add<0x4E>(x);   // quad_perm: lane ^ 2
  x = dpp_add<0x141>(x);  // mirror of eight: the other quad
  if constexpr (N == 16) x = dpp_add<0x140>(x);  // mirror of sixteen: the other eight
  return x;
}

__device__ __forceinline__ uint32_t round_pair(float a, float b) {
  const f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

template <int D, HeadNorm NORM, bool HALF>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(QkNormRopeParams p, uint32_t units, uint32_t q_units) {
  constexpr int LANES = D / 8, ROWS = 256 / LANES;
  // The units (side, kHeads heads) of a row on one XCD, one after another: its table rows come from that L2 then.
  const uint32_t in_xcd = blockIdx.x >> 3, unit = in_xcd % units;
  const int64_t row = ((int64_t)(in_xcd / units) * 8 + (blockIdx.x & 7)) * ROWS + threadIdx.x / LANES;
  if (row >= p.n_rows) return;
  const bool keys = unit >= q_units;
  const NormHeadsParams& s = p.side[keys ? 1 : 0];
  const int h0 = (int)(keys ? unit - q_units : unit) * kHeads;
  const int t = threadIdx.x % LANES;
  const bool turned = t < p.rot_dim / 8;
  // Elements of this lane: four from e0, four from e1.
  const int e0 = HALF && turned ? 4 * t : 8 * t;
  const int e1 = HALF && turned ? p.rot_dim / 2 + 4 * t : 8 * t + 4;

  const char* src = s.x + row * s.row_stride_b + (int64_t)h0 * (2 * D);
  u32x2 in[kHeads][2];
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    if (h0 + i < s.n_heads) {
      if constexpr (HALF) {
        in[i][0] = *reinterpret_cast<const u32x2*>(src + i * 2 * D + 2 * e0);
        in[i][1] = *reinterpret_cast<const u32x2*>(src + i * 2 * D + 2 * e1);
      } else {
        const u32x4 w = *reinterpret_cast<const u32x4*>(src + i * 2 * D + 2 * e0);
        in[i][0] = u32x2{w[0], w[1]};
        in[i][1] = u32x2{w[2], w[3]};
      }
    }
  }
  float c[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
  if (turned) {
    const f32x4* tab = reinterpret_cast<const f32x4*>(p.table + row * p.rot_dim + 8 * t);
    const f32x4 a = tab[0], b = tab[1];
    c[0] = a[0]; sn[0] = a[1]; c[1] = a[2]; sn[1] = a[3];
    c[2] = b[0]; sn[2] = b[1]; c[3] = b[2]; sn[3] = b[3];
  }
  float w[8], bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    w[e] = 1.f;
    bias[e] = 0.f;
  }
  if (NORM != HeadNorm::kNone && s.weight != nullptr) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(s.weight + e0), b = *reinterpret_cast<const f32x4*>(s.weight + e1);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = a[e];
      w[4 + e] = b[e];
    }
  }
  if (NORM != HeadNorm::kNone && s.bias != nullptr) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(s.bias + e0), b = *reinterpret_cast<const f32x4*>(s.bias + e1);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bias[e] = a[e];
      bias[4 + e] = b[e];
    }
  }
  char* dst = s.out + row * s.out_stride_b + (int64_t)h0 * (2 * D);
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    if (h0 + i >= s.n_heads) break;
    float y[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      y[2 * k] = __builtin_bit_cast(float, in[i][k >> 1][k & 1] << 16);
      y[2 * k + 1] = __builtin_bit_cast(float, in[i][k >> 1][k & 1] & 0xFFFF0000u);
    }
    if constexpr (NORM == HeadNorm::kLayer) {
      const float mean = group_sum<LANES>(((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]))) * (1.f / D);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] -= mean;
    }
    if constexpr (NORM != HeadNorm::kNone) {
      float sq = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sq = __builtin_fmaf(y[e], y[e], sq);
      const float r = 1.f / __builtin_sqrtf(group_sum<LANES>(sq) * (1.f / D) + p.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = __builtin_fmaf(y[e] * r, w[e], bias[e]);
    }
    if (turned) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float &a = y[HALF ? k : 2 * k], &b = y[HALF ? 4 + k : 2 * k + 1];
        const float a1 = a * c[k] - b * sn[k], b1 = b * c[k] + a * sn[k];
        a = a1;
        b = b1;
      }
    }
    const u32x2 o0 = {round_pair(y[0], y[1]), round_pair(y[2], y[3])}, o1 = {round_pair(y[4], y[5]), round_pair(y[6], y[7])};
    if constexpr (HALF) {
      *reinterpret_cast<u32x2*>(dst + i * 2 * D + 2 * e0) = o0;
      *reinterpret_cast<u32x2*>(dst + i * 2 * D + 2 * e1) = o1;
    } else {
      *reinterpret_cast<u32x4*>(dst + i * 2 * D + 2 * e0) = u32x4{o0[0], o0[1], o1[0], o1[1]};
    }
  }
}

static uint32_t units_of(const NormHeadsParams& s) { return ((uint32_t)s.n_heads + kHeads - 1) / kHeads; }

int64_t qk_norm_rope_blocks(const QkNormRopeParams& p, int head_dim) {
  const int64_t rows = 256 / (head_dim / 8), row_blocks = (p.n_rows + rows - 1) / rows;
  return (row_blocks + 7) / 8 * 8 * (units_of(p.side[0]) + units_of(p.side[1]));
}

template <int D, HeadNorm NORM, bool HALF>
static void launch(const QkNormRopeParams& p, hipStream_t stream) {
  const uint32_t q_units = units_of(p.side[0]), units = q_units + units_of(p.side[1]);
  hipLaunchKernelGGL((qk_norm_rope_kernel<D, NORM, HALF>), dim3((unsigned)qk_norm_rope_blocks(p, D)), dim3(256), 0, stream, p, units, q_units);
}
template <int D, HeadNorm NORM>
static void launch_layout(const QkNormRopeParams& p, hipStream_t stream) {
  p.half ? launch<D, NORM, true>(p, stream) : launch<D, NORM, false>(p, stream);
}
template <int D>
static void launch_norm(const QkNormRopeParams& p, HeadNorm norm, hipStream_t stream) {
  if (norm == HeadNorm::kNone) launch_layout<D, HeadNorm::kNone>(p, stream);
  else if (norm == HeadNorm::kRms) launch_layout<D, HeadNorm::kRms>(p, stream);
  else launch_layout<D, HeadNorm::kLayer>(p, stream);
}

hipError_t qk_norm_rope_launch(const QkNormRopeParams& p, HeadNorm norm, int head_dim, hipStream_t stream) {
  if (p.n_rows == 0) return hipSuccess;
  head_dim == 64 ? launch_norm<64>(p, norm, stream) : launch_norm<128>(p, norm, stream);
  return hipGetLastError();
}

}  // namespace dit
