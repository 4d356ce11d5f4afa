// Linear layers on few rows (a decoding step): what bounds them is reading every weight once, so the weights go
// straight from memory into the MFMA operand registers, no LDS and no barrier between them, with as many loads in
// flight as registers hold.
//
// A workgroup has 16 filters (gated: 16 of the gate and the same 16 of the layer it gates) and MT * 16 rows; its WK
// waves take the reduction in turns of 128 bytes of every row.  Lane l reads 32 consecutive bytes of filter l % 16:
// four lanes a whole line.  Rows beyond the last one and bytes beyond the reduction's end are fetched from outside
// the buffer's range, which brings zeros and no traffic.  The waves' sums meet in LDS and are added in the waves' order.
#include <hip/hip_runtime.h>

#include "linear_device.h"
#include "tuning.h"

namespace fupr {

fupr_status launch_status(const char* what);

namespace {

constexpr uint32_t kOutside = 0x80000000u;
constexpr int kAhead = 4;   // steps whose loads are in flight together

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint4 load16(const __amdgpu_buffer_rsrc_t& r, uint32_t off) {
  return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0));
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const char* base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, (int)kOutside, 0x00020000);
}

template <int TY, bool GATED, int MT, int WK>
__global__ __launch_bounds__(WK * 64) void linear_rows_kernel(LinearParams p) {
  constexpr int NT = GATED ? 2 : 1, PER = 16 / elem_bytes<TY>(), STEP = 8 * PER;   // elements of a chunk, of a step
  __shared__ __attribute__((aligned(16))) f32x4 part[WK][MT * NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, g = lane >> 4;
  int e = 0, hi = p.M, m0, n_len = p.N, k_len = p.K;
  const int mt_at = blockIdx.x / p.n_tiles, n0 = (blockIdx.x - mt_at * p.n_tiles) * 16;
  if (p.offsets) {
    ExpertRows r;
    if (!find_expert<MT * 16>(p, mt_at, lane, r)) return;
    e = r.e;
    hi = r.hi;
    m0 = r.lo + r.tile * MT * 16;
    n_len = r.n_len;
    k_len = r.k_len;
  } else {
    m0 = mt_at * MT * 16;
  }
  const int steps = n0 < n_len ? (k_len + STEP - 1) / STEP : 0;
  const int chunks = (k_len + PER - 1) / PER;

  const char* w0 = p.w + e * p.w_expert + n0 * p.w_stride;
  const __amdgpu_buffer_rsrc_t wr = rsrc_of(w0);
  const __amdgpu_buffer_rsrc_t ur = rsrc_of(GATED ? p.w_up + e * p.w_expert + n0 * p.w_stride : w0);
  const __amdgpu_buffer_rsrc_t xr = rsrc_of(p.x);
  const uint32_t woff = n0 + li < n_len ? (uint32_t)(li * p.w_stride) : kOutside;
  uint32_t xoff[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int row = m0 + mt * 16 + li;
    int from = row;
    if (p.src && row < hi) from = min(max(p.src[row], 0), p.x_rows - 1);
    xoff[mt] = row < hi ? (uint32_t)(from * p.x_stride) : kOutside;
  }

  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = zero;

  for (int s0 = wave; s0 < steps; s0 += WK * kAhead) {
    uint4 a[kAhead][NT][2], b[kAhead][MT][2];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int chunk = (s0 + u * WK) * 8 + g * 2 + h;
        const uint32_t beyond = chunk < chunks ? 0u : kOutside, at = (uint32_t)chunk * 16u;
        a[u][0][h] = load16(wr, (woff + at) | beyond);
        if constexpr (GATED) a[u][1][h] = load16(ur, (woff + at) | beyond);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) b[u][mt][h] = load16(xr, (xoff[mt] + at) | beyond);
      }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int s = s0 + u * WK;
      if (s * STEP < k_len && (s + 1) * STEP > k_len) {   // the step in which the reduction ends
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int valid = k_len - (s * 8 + g * 2 + h) * PER;
#pragma unroll
          for (int j = 0; j < NT; ++j) a[u][j][h] = keep_first<TY>(a[u][j][h], valid);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) b[u][mt][h] = keep_first<TY>(b[u][mt][h], valid);
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[mt][j] = mfma_chunks<TY>(a[u][j][h], b[u][mt][h], acc[mt][j]);
    }
  }

#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int j = 0; j < NT; ++j) part[wave][mt * NT + j][lane] = acc[mt][j];
  __syncthreads();
  constexpr bool FINE = TY == FUPR_F32;
  const int n = n0 + g * 4;
  const int64_t bias_at = (int64_t)e * p.N + n;
  for (int mt = wave; mt < MT; mt += WK) {
    const int row = m0 + mt * 16 + li;
    if (row >= hi) continue;
    f32x4 v = zero, up = zero;
#pragma unroll
    for (int k = 0; k < WK; ++k) {
      v += part[k][mt * NT][lane];
      if constexpr (GATED) up += part[k][mt * NT + 1][lane];
    }
    float out[4];
    with_activation(p.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool there = n + i < n_len;
        float h = activate<FINE, decltype(act)::value>(v[i] + (p.bias && there ? p.bias[bias_at + i] : 0.f));
        if constexpr (GATED) h *= up[i] + (p.bias_up && there ? p.bias_up[bias_at + i] : 0.f);
        out[i] = there ? h : 0.f;
      }
    });
    store_run<TY, 4>(p, row, n, out);
  }
}

template <int TY, bool GATED, int MT>
fupr_status launch_as(LinearParams p, hipStream_t st) {
  constexpr int WK = 8;
  p.n_tiles = (p.N + 15) / 16;
  const int BM = MT * 16;
  if (p.offsets) {
    const int begun = p.E < p.M ? p.E : p.M;
    p.m_tiles = begun + (p.M - begun) / BM;
  } else {
    p.m_tiles = (p.M + BM - 1) / BM;
  }
  const int64_t blocks = (int64_t)p.m_tiles * p.n_tiles;
  if (blocks > 0x7fffffff) return FUPR_ERR_LIMIT;
  linear_rows_kernel<TY, GATED, MT, WK><<<dim3((unsigned)blocks), dim3(WK * 64), 0, st>>>(p);
  return launch_status("linear_rows_kernel");
}

// Rows of a layer, or of the average expert that can have any.
int rows_of(const LinearParams& p) { return p.offsets ? (p.M + p.E - 1) / p.E : p.M; }

template <int TY, bool GATED>
fupr_status launch_rows(const LinearParams& p, hipStream_t st) {
  const int rows = rows_of(p);
  if (rows <= 16) return launch_as<TY, GATED, 1>(p, st);
  if (rows <= 32) return launch_as<TY, GATED, 2>(p, st);
  return launch_as<TY, GATED, 4>(p, st);
}

template <int TY>
fupr_status launch_type(const LinearParams& p, hipStream_t st) {
  return p.w_up ? launch_rows<TY, true>(p, st) : launch_rows<TY, false>(p, st);
}

}  // namespace

bool linear_rows_applies(const LinearParams& p, fupr_dtype dt) {
  (void)dt;
  int most = tuning_any() ? tuning_int("linear_rows", -1) : -1;
  if (most < 0) most = 64;
  // sixteen filters and all of x are reached with 31-bit offsets
  const int64_t limit = int64_t(1) << 31;
  return rows_of(p) <= most && 16 * p.w_stride <= limit && p.x_rows * p.x_stride <= limit;
}

fupr_status launch_linear_rows(LinearParams p, fupr_dtype dt, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  switch (dt) {
    case FUPR_BF16: return launch_type<FUPR_BF16>(p, st);
    case FUPR_F16: return launch_type<FUPR_F16>(p, st);
    default: return launch_type<FUPR_F32>(p, st);
  }
}

}  // namespace fupr
