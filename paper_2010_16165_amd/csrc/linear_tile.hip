// Linear layers on many rows, one layer or one per expert: y = a(x W^T + b) (* (x Wu^T + bu)) (+ res), a matrix
// product in tiles of BM rows x BN filters.  Both operands have the reduction along their rows in memory, so a step
// of 128 bytes of every row of the tile goes global -> LDS as it lies (asynchronous loads of 16 bytes per lane that
// need no registers), a ring of D buffers keeping D - 1 steps in flight.
//
// LDS row r holds its eight 16-byte chunks at chunk ^ (r / 2 & 7): the lanes of an operand read (16 rows, 128 bytes
// apart, one chunk) then cover all 64 banks once.  Filters are MFMA operand A, rows of x operand B, so a lane ends up with four filters'
// results of one row; which filter an LDS row holds is chosen such that a lane's tiles together are consecutive
// columns of y (16-byte stores).  A gated layer alternates tiles of the gate and of the layer that it gates: both
// results of a column meet in one lane.
#include <hip/hip_runtime.h>

#include "linear_device.h"
#include "tuning.h"

namespace fupr {

fupr_status launch_status(const char* what);

namespace {

// 64 lanes x 16 bytes from their own addresses to 1024 consecutive bytes of LDS
__device__ __forceinline__ void load_to_lds(const char* from, uint32_t lds_base) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off"
      :
      : "s"(lds_base), "v"(from)
      : "memory", "m0");
}

template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <int TY_, int WM_, int WN_, int MT_, int NT_, int D_>
struct TileGeom {
  static constexpr int TY = TY_, WM = WM_, WN = WN_, MT = MT_, NT = NT_, D = D_;
  static constexpr int waves = WM * WN, threads = waves * 64;
  static constexpr int BM = WM * MT * 16, BN = WN * NT * 16;
  static constexpr int xl = BM / 8 / waves, wl = BN / 8 / waves;   // loads of a wave and step (8 rows each)
  static_assert(xl * 8 * waves == BM && wl * 8 * waves == BN && NT % 2 == 0, "whole loads, pairs of tiles");
  static constexpr int buf = (BM + BN) * 128;
  static constexpr int per_chunk = 16 / elem_bytes<TY>(), per_step = 8 * per_chunk;
};

template <class G, bool GATED>
__device__ __forceinline__ void tile_epilogue(const LinearParams& p, f32x4 (&acc)[G::MT][G::NT], int e, int hi, int row0,
                                              int nb, int n_len, int lane) {
  constexpr int NT = G::NT, MT = G::MT, Q = GATED ? NT / 2 : NT;   // four-column pieces of a lane
  constexpr bool FINE = G::TY == FUPR_F32;
  const int n0 = nb + (lane >> 4) * 4 * Q;
  const float* b = p.bias ? p.bias + (int64_t)e * p.N : nullptr;
  const float* bu = p.bias_up ? p.bias_up + (int64_t)e * p.N : nullptr;
  auto add = [&](const float* from, int first, int step) {
    if (!from) return;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = n0 + q * 4 + i;
        const float v = n < n_len ? from[n] : 0.f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[mt][first + q * step][i] += v;
      }
  };
  add(b, 0, GATED ? 2 : 1);
  if constexpr (GATED) add(bu, 1, 2);
  with_activation(p.act, [&](auto act) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v = activate<FINE, decltype(act)::value>(acc[mt][GATED ? 2 * q : q][i]);
          if constexpr (GATED) v *= acc[mt][2 * q + 1][i];
          acc[mt][GATED ? 2 * q : q][i] = v;
        }
  });
  if (nb + 4 * Q * 4 > n_len) {   // columns that pruning took from this expert
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n0 + q * 4 + i >= n_len)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) acc[mt][GATED ? 2 * q : q][i] = 0.f;
  }
  constexpr int kPer = Q % 2 ? 1 : 2;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int row = row0 + mt * 16 + (lane & 15);
    if (row >= hi) continue;
#pragma unroll
    for (int q = 0; q < Q; q += kPer) {
      float v[4 * kPer];
#pragma unroll
      for (int i = 0; i < 4 * kPer; ++i) v[i] = acc[mt][GATED ? 2 * (q + i / 4) : q + i / 4][i & 3];
      store_run<G::TY, 4 * kPer>(p, row, n0 + q * 4, v);
    }
  }
}

template <class G>
__global__ __launch_bounds__(G::threads) void linear_tile_kernel(LinearParams p) {
  constexpr int BM = G::BM, BN = G::BN, MT = G::MT, NT = G::NT, D = G::D;
  __shared__ __attribute__((aligned(1024))) char lds[D * G::buf];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool gated = p.w_up != nullptr;
  const int cols = gated ? BN / 2 : BN;   // of y, in a tile

  int e = 0, hi = p.M, m0, nt, n_len = p.N, k_len = p.K;
  if (p.offsets) {
    const int at = tile_of_workgroup(blockIdx.x, count_expert_tiles<BM>(p, lane) * p.n_tiles);
    if (at < 0) return;
    ExpertRows r;
    const int mt = at / p.n_tiles;
    nt = at - mt * p.n_tiles;
    if (!find_expert<BM>(p, mt, lane, r)) return;
    e = r.e;
    hi = r.hi;
    m0 = r.lo + r.tile * BM;
    n_len = r.n_len;
    k_len = r.k_len;
  } else {
    // strips of eight row tiles: what an XCD holds at one time is about as tall as it is wide
    const int at = tile_of_workgroup(blockIdx.x, p.m_tiles * p.n_tiles);
    if (at < 0) return;
    const int strip = at / (8 * p.n_tiles), tall = min(8, p.m_tiles - strip * 8);
    const int in = at - strip * 8 * p.n_tiles;
    nt = in / tall;
    m0 = (strip * 8 + in - nt * tall) * BM;
  }
  const int n0 = nt * cols;
  const int steps = n0 < n_len ? (k_len + G::per_step - 1) / G::per_step : 0;

  // the lane's place in every load: row lane / 8 of eight, and the chunk that is kept there
  static_assert(G::waves % 2 == 0, "the eight rows of a wave's loads are always even or always odd ones");
  const int chunk = (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4));
  constexpr int kLoads = G::xl + G::wl;
  const char* from[kLoads];
#pragma unroll
  for (int i = 0; i < G::xl; ++i) {
    int row = min(m0 + (i * G::waves + wave) * 8 + (lane >> 3), hi - 1);
    if (p.src) row = min(max(p.src[row], 0), p.x_rows - 1);
    from[i] = p.x + row * p.x_stride + chunk * 16;
  }
#pragma unroll
  for (int i = 0; i < G::wl; ++i) {
    const int r = (i * G::waves + wave) * 8 + (lane >> 3);
    const int wn = r / (NT * 16), t = (r >> 4) % NT, j = r & 15;
    const int n = gated ? n0 + wn * NT * 8 + (j >> 2) * 2 * NT + 4 * (t >> 1) + (j & 3)
                        : n0 + wn * NT * 16 + (j >> 2) * 4 * NT + 4 * t + (j & 3);
    const char* w = gated && (t & 1) ? p.w_up : p.w;
    from[G::xl + i] = w + e * p.w_expert + min(n, max(n_len, 1) - 1) * p.w_stride + chunk * 16;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

  // Loads of one step after the other into buffer after buffer.  In the step that the reduction ends in, chunks behind
  // its last one are that last one again (inside the row, and zeroed below).
  uint32_t to = lds0 + wave * 1024;
  int issued = 0;
  auto issue = [&]() {
    if (++issued == steps) {
      const int last = (k_len + G::per_chunk - 1) / G::per_chunk - 1;
      const int back = max((steps - 1) * 8 + chunk - last, 0) * 16;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) from[i] -= back;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      load_to_lds(from[i], to + i * G::waves * 1024);
      from[i] += 128;
    }
    to += G::buf;
    if (to >= lds0 + D * G::buf) to -= D * G::buf;
  };

  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = zero;

  const int wm = wave / G::WN, wn = wave % G::WN;
  const int at0 = (lane & 15) * 128 + ((lane >> 4) ^ (lane >> 1 & 7)) * 16;
#pragma unroll
  for (int s = 0; s < D - 1; ++s)
    if (s < steps) issue();
  int buf = 0;
  for (int s = 0; s < steps; ++s) {
    if (s + D - 1 <= steps) wait_loads<(D - 2) * kLoads>();
    else wait_loads<0>();
    const int left = k_len - s * G::per_step;
    if (left < G::per_step) {
      // the last step of a reduction that does not fill it: zeros behind its end, in the wave's own part
      const int valid = left - chunk * G::per_chunk;
      if (valid < G::per_chunk) {
        char* mine = lds + buf + wave * 1024 + lane * 16;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          uint4* v = reinterpret_cast<uint4*>(mine + i * G::waves * 1024);
          *v = keep_first<G::TY>(*v, valid);
        }
      }
    }
    __syncthreads();
    if (s + D - 1 < steps) issue();
    const char* xs = lds + buf + wm * MT * 2048;
    const char* ws = lds + buf + BM * 128 + wn * NT * 2048;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int at = at0 ^ (half * 64);
      uint4 a[NT], b[MT];
#pragma unroll
      for (int j = 0; j < NT; ++j) a[j] = *reinterpret_cast<const uint4*>(ws + j * 2048 + at);
#pragma unroll
      for (int i = 0; i < MT; ++i) b[i] = *reinterpret_cast<const uint4*>(xs + i * 2048 + at);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = mfma_chunks<G::TY>(a[j], b[i], acc[i][j]);
    }
    buf = buf + G::buf == D * G::buf ? 0 : buf + G::buf;
  }

  const int row0 = m0 + wm * MT * 16;
  if (gated) tile_epilogue<G, true>(p, acc, e, hi, row0, n0 + wn * NT * 8, n_len, lane);
  else tile_epilogue<G, false>(p, acc, e, hi, row0, n0 + wn * NT * 16, n_len, lane);
}

template <class G>
fupr_status launch_as(LinearParams p, hipStream_t st) {
  const int cols = p.w_up ? G::BN / 2 : G::BN;
  p.n_tiles = (p.N + cols - 1) / cols;
  if (p.offsets) {
    // at most: one tile begun by every expert that can have a row, the others full
    const int begun = p.E < p.M ? p.E : p.M;
    p.m_tiles = begun + (p.M - begun) / G::BM;
  } else {
    p.m_tiles = (p.M + G::BM - 1) / G::BM;
  }
  const int64_t tiles = (int64_t)p.m_tiles * p.n_tiles;
  if (tiles > 0x7fffff00) return FUPR_ERR_LIMIT;
  linear_tile_kernel<G><<<dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(G::threads), 0, st>>>(p);
  return launch_status("linear_tile_kernel");
}

template <int TY>
fupr_status launch_type(const LinearParams& p, hipStream_t st) {
  switch (tuning_any() ? tuning_int("linear_tile", 0) : 0) {
    case 1: return launch_as<TileGeom<TY, 2, 4, 8, 4, 2>>(p, st);
    case 2: return launch_as<TileGeom<TY, 2, 4, 4, 4, 3>>(p, st);
    case 3: return launch_as<TileGeom<TY, 2, 2, 2, 2, 4>>(p, st);
    case 4: return launch_as<TileGeom<TY, 2, 2, 8, 8, 2>>(p, st);
    case 5: return launch_as<TileGeom<TY, 2, 2, 4, 4, 2>>(p, st);
    case 6: return launch_as<TileGeom<TY, 2, 2, 2, 4, 3>>(p, st);
    default: return launch_as<TileGeom<TY, 2, 2, 4, 4, 3>>(p, st);
  }
}

}  // namespace

fupr_status launch_linear_tile(LinearParams p, fupr_dtype dt, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  switch (dt) {
    case FUPR_BF16: return launch_type<FUPR_BF16>(p, st);
    case FUPR_F16: return launch_type<FUPR_F16>(p, st);
    default: return launch_type<FUPR_F32>(p, st);
  }
}

}  // namespace fupr
