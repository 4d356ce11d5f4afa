// Internal: what the kernels of linear layers share - element types, which tile a workgroup has, the epilogue.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "device_utils.h"
#include "linear.h"

namespace fupr {

// TY below is the fupr_dtype of x and the weights.
template <int TY>
constexpr int elem_bytes() {
  return TY == FUPR_F32 ? 4 : 2;
}

// Sixteen filters x sixteen rows x one 16-byte chunk per lane (lane l: filter or row l % 16, chunk l / 16 of four).
// In single precision four instructions take one element of every lane's chunk each: the order in which a sum's
// products are taken is free as long as both operands keep to it.
template <int TY>
__device__ __forceinline__ f32x4 mfma_chunks(const uint4& a, const uint4& b, f32x4 c) {
  if constexpr (TY == FUPR_F32) {
    c = mfma_16x16x4(a.x, b.x, c);
    c = mfma_16x16x4(a.y, b.y, c);
    c = mfma_16x16x4(a.z, b.z, c);
    return mfma_16x16x4(a.w, b.w, c);
  } else {
    return mfma_16x16x32<TY == FUPR_BF16>(a, b, c);
  }
}

// The first `valid` elements of a chunk, zeros behind them.
template <int TY>
__device__ __forceinline__ uint4 keep_first(uint4 v, int valid) {
  uint32_t d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (TY == FUPR_F32) {
      d[i] = i < valid ? d[i] : 0u;
    } else {
      const int left = valid - 2 * i;
      d[i] = left >= 2 ? d[i] : left == 1 ? d[i] & 0xffffu : 0u;
    }
  }
  return uint4{d[0], d[1], d[2], d[3]};
}

// e^v by the hardware's 2^v for results of 16 bits (its error, 2^-22 and |v| 2^-24 relative, is far below their half
// step), the library's for single precision.
template <bool FINE>
__device__ __forceinline__ float exp_of(float v) {
  if constexpr (FINE) return expf(v);
  return __builtin_amdgcn_exp2f(v * 1.4426950408889634f);
}

// erfc(z) for z >= 0: e^(-z z) t Q(t) with t = 1 / (1 + 0.38 z), Q of degree 8 fitted to erfc(z) e^(z z) over 0 .. 14 by
// reweighted least squares in relative error (2.5e-8; 4e-7 with its fp32 rounding).  Beyond 14 the exponential is 0.
template <bool FINE>
__device__ __forceinline__ float erfc_of(float z) {
  float t, tail = 0.f;
  const float zz = z * z;
  if constexpr (FINE) {
    t = 1.f / (1.f + 0.38f * z);
    tail = z < 14.f ? fmaf(z, z, -zz) : 0.f;   // what rounding took from z z
  } else {
    t = __builtin_amdgcn_rcpf(1.f + 0.38f * z);
  }
  float q = 0.058422474f;
  q = fmaf(q, t, -0.25986333f);
  q = fmaf(q, t, 0.35934416f);
  q = fmaf(q, t, -0.15684429f);
  q = fmaf(q, t, 0.22722182f);
  q = fmaf(q, t, 0.13967941f);
  q = fmaf(q, t, 0.20368547f);
  q = fmaf(q, t, 0.21394443f);
  q = fmaf(q, t, 0.21440983f);
  return q * t * exp_of<FINE>(-zz) * (1.f - tail);
}

// None of these takes a difference of nearly equal numbers: v Phi(v) from the upper tail, both sigmoid forms as a
// quotient.  At -inf they are NaN but for the first two, as their formulas.
template <bool FINE, int ACT>
__device__ __forceinline__ float activate(float v) {
  if constexpr (ACT == FUPR_ACT_NONE) {
    return v;
  } else if constexpr (ACT == FUPR_ACT_RELU) {
    return v < 0.f ? 0.f : v;
  } else if constexpr (ACT == FUPR_ACT_GELU) {
    const float upper = 0.5f * erfc_of<FINE>(fabsf(v) * 0.70710678118654752f);
    return v * (v < 0.f ? upper : 1.f - upper);
  } else {
    const float u = ACT == FUPR_ACT_SILU ? v : 1.5957691216057308f * v * (1.f + 0.044715f * v * v);
    const float d = 1.f + exp_of<FINE>(-u);
    if constexpr (FINE) return v / d;
    return v * __builtin_amdgcn_rcpf(d);
  }
}
// f(integral_constant of the activation): the choice is made once for a tile, not once for every element.
template <int ACT>
struct ActTag {
  static constexpr int value = ACT;
};
template <class F>
__device__ __forceinline__ void with_activation(int act, F f) {
  switch (act) {
    case FUPR_ACT_NONE: f(ActTag<FUPR_ACT_NONE>{}); break;
    case FUPR_ACT_RELU: f(ActTag<FUPR_ACT_RELU>{}); break;
    case FUPR_ACT_SILU: f(ActTag<FUPR_ACT_SILU>{}); break;
    case FUPR_ACT_GELU: f(ActTag<FUPR_ACT_GELU>{}); break;
    default: f(ActTag<FUPR_ACT_GELU_TANH>{});
  }
}

// The row tiles of experts: which expert has tile `at`, and how many tiles there are.  Every lane returns the same.
// A wave counts 64 experts at a time; an expert's rows are what its two offsets, clamped into 0 .. M, span.
struct ExpertRows {
  int e, lo, hi, tile;   // tile: of the expert's own
  int n_len, k_len;
};
template <int BM>
__device__ __forceinline__ int expert_tiles(const LinearParams& p, int e, int& lo, int& hi) {
  lo = hi = 0;
  if (e < p.E) {
    lo = min(max(p.offsets[e], 0), p.M);
    hi = min(max(p.offsets[e + 1], lo), p.M);
  }
  return (hi - lo + BM - 1) / BM;
}
__device__ __forceinline__ int wave_prefix(int v, int lane) {   // inclusive
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}
template <int BM>
__device__ __forceinline__ int count_expert_tiles(const LinearParams& p, int lane) {
  int total = 0;
  for (int e0 = 0; e0 < p.E; e0 += 64) {
    int lo, hi;
    total += __shfl(wave_prefix(expert_tiles<BM>(p, e0 + lane, lo, hi), lane), 63);
  }
  return __builtin_amdgcn_readfirstlane(total);
}
template <int BM>
__device__ __forceinline__ bool find_expert(const LinearParams& p, int at, int lane, ExpertRows& out) {
  int before = 0;
  for (int e0 = 0; e0 < p.E; e0 += 64) {
    int lo, hi;
    const int n = expert_tiles<BM>(p, e0 + lane, lo, hi);
    // (asked for together with the offsets: one latency, not two)
    const int mine_n = p.n_len && e0 + lane < p.E ? p.n_len[e0 + lane] : p.N;
    const int mine_k = p.k_len && e0 + lane < p.E ? p.k_len[e0 + lane] : p.K;
    const int upto = before + wave_prefix(n, lane);
    const uint64_t mine = __ballot(at >= upto - n && at < upto);
    if (mine) {
      const int who = __builtin_ctzll(mine);
      out.e = __builtin_amdgcn_readfirstlane(e0 + who);
      out.lo = __builtin_amdgcn_readfirstlane(__shfl(lo, who));
      out.hi = __builtin_amdgcn_readfirstlane(__shfl(hi, who));
      out.tile = __builtin_amdgcn_readfirstlane(at - __shfl(upto - n, who));
      out.n_len = __builtin_amdgcn_readfirstlane(min(max(__shfl(mine_n, who), 0), p.N));
      out.k_len = __builtin_amdgcn_readfirstlane(min(max(__shfl(mine_k, who), 0), p.K));
      return true;
    }
    before = __shfl(upto, 63);
  }
  return false;
}

// Workgroups go to the eight XCDs in turn; tile numbers are handed out so that an XCD takes a contiguous range of
// `total` tiles and its L2 sees neighbours.  -1: this workgroup has none.
__device__ __forceinline__ int tile_of_workgroup(int id, int total) {
  const int each = (total + 7) >> 3;
  const int at = (id & 7) * each + (id >> 3);
  return (id >> 3) < each && at < total ? at : -1;
}

// COUNT consecutive results (4 or 8) of one row from column n on: + res, one rounding, stored with 16-byte accesses
// where the row still has that many columns.
template <int TY, int COUNT>
__device__ __forceinline__ void store_run(const LinearParams& p, int64_t row, int n, float* v) {
  if (n >= p.N) return;
  const bool whole = n + COUNT <= p.N;
  const int es = TY == FUPR_F32 || p.y_f32 ? 4 : 2;
  char* y = p.y + row * p.y_stride + (int64_t)n * es;
  const char* res = p.res ? p.res + row * p.res_stride + (int64_t)n * es : nullptr;
  if (TY == FUPR_F32 || p.y_f32) {
    if (whole) {
#pragma unroll
      for (int i = 0; i < COUNT; i += 4) {
        f32x4 r = {0.f, 0.f, 0.f, 0.f};
        if (res) r = *reinterpret_cast<const f32x4*>(res + i * 4);
        *reinterpret_cast<f32x4*>(y + i * 4) = f32x4{v[i] + r[0], v[i + 1] + r[1], v[i + 2] + r[2], v[i + 3] + r[3]};
      }
    } else {
#pragma unroll
      for (int i = 0; i < COUNT; ++i)
        if (n + i < p.N)
          reinterpret_cast<float*>(y)[i] = v[i] + (res ? reinterpret_cast<const float*>(res)[i] : 0.f);
    }
  } else {
    constexpr bool BF = TY == FUPR_BF16;
    if (whole) {
      uint32_t r[COUNT / 2] = {}, o[COUNT / 2];
      if (res) {
#pragma unroll
        for (int i = 0; i < COUNT / 4; ++i) {
          const uint2 q = *reinterpret_cast<const uint2*>(res + i * 8);
          r[2 * i] = q.x;
          r[2 * i + 1] = q.y;
        }
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] += to_float<BF>((uint16_t)(r[i / 2] >> (i & 1) * 16));
      }
#pragma unroll
      for (int i = 0; i < COUNT / 2; ++i) o[i] = pack2<BF>(v[2 * i], v[2 * i + 1]);
      if constexpr (COUNT == 8) *reinterpret_cast<uint4*>(y) = uint4{o[0], o[1], o[2], o[3]};
      else *reinterpret_cast<uint2*>(y) = uint2{o[0], o[1]};
    } else {
#pragma unroll
      for (int i = 0; i < COUNT; ++i)
        if (n + i < p.N)
          reinterpret_cast<uint16_t*>(y)[i] =
              from_float<BF>(v[i] + (res ? to_float<BF>(reinterpret_cast<const uint16_t*>(res)[i]) : 0.f));
    }
  }
}

}  // namespace fupr
