// Linear layers on very many rows, 16-bit types: tiles of 256 rows x 256 filters on eight waves of 128 x 64.
//
// Why so large: a compute unit takes in 64 bytes per clock, and 128 x 128 tiles need that much to keep the matrix
// units busy; these need half.  A step of 128 bytes of every row (64 elements, whole lines) goes global -> LDS as in
// linear_tile.hip, two buffers of 64 KB.
//
// The waves' halves take turns: while the first four (one per SIMD) multiply a step from registers, the other four
// read theirs from LDS, all of it, 96 registers beside 128 of accumulators.  Each phase ends in a barrier; in it one
// half does nothing but multiply, at a raised wave priority.  Phase 2 s: the first half reads step s, the second
// multiplies s - 1, and both ask for step s + 1 into the buffer that the second half has read to its end in phase
// 2 s - 1; it has landed when phase 2 s + 1 ends.
//
// LDS row r (128 bytes) holds its eight chunks at chunk ^ (r / 2 & 7): operand reads cover all 64 banks once.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "linear_tile.h"

namespace fupr {

fupr_status launch_status(const char* what);

namespace {

constexpr int BM = 256, BN = 256, MT = 8, NT = 4, kWaves = 8, kLoads = 8;   // loads: of a wave and step, 8 rows each
constexpr int kBuf = (BM + BN) * 128;

// The end of a phase: what this wave read from LDS has arrived, and no wave goes on before all have come here.
__device__ __forceinline__ void phase_ends() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// 64 lanes x 16 bytes from base + their offset to 1024 consecutive bytes of LDS
__device__ __forceinline__ void load_to_lds_from(const char* base, uint32_t off, uint32_t lds_base) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %2"
      :
      : "s"(lds_base), "v"(off), "s"(base)
      : "memory", "m0");
}

__device__ __forceinline__ uint4 read_lds(uint32_t at) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(uint4, *(const u32x4 __attribute__((address_space(3)))*)(uintptr_t)at);
}

template <int TY>
__global__ __launch_bounds__(kWaves * 64, 2) void linear_wide_kernel(LinearParams p) {
  constexpr int kChunk = 8, kStep = 64;   // elements
  __shared__ __attribute__((aligned(1024))) char lds[2 * kBuf];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool gated = p.w_up != nullptr;
  TilePlace at;
  if (!find_tile<BM>(p, lane, at)) return;
  const int e = at.e, hi = at.hi, m0 = at.m0, n_len = at.n_len, k_len = at.k_len;
  const int n0 = at.nt * (gated ? BN / 2 : BN);
  const int steps = n0 < n_len ? (k_len + kStep - 1) / kStep : 0;

  // the lane's place in every load: row lane / 8 of eight, and the chunk that is kept there
  const int chunk = (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4));
  uint32_t off[kLoads];
  const char* xb = p.src ? p.x : p.x + (int64_t)m0 * p.x_stride;
  const char* wb = p.w + e * p.w_expert + n0 * p.w_stride;
  const char* ub = gated ? p.w_up + e * p.w_expert + n0 * p.w_stride : wb;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = min(m0 + (i * kWaves + wave) * 8 + (lane >> 3), hi - 1);
    const int from = p.src ? min(max(p.src[row], 0), p.x_rows - 1) : row - m0;
    off[i] = (uint32_t)from * (uint32_t)p.x_stride + chunk * 16;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = min(filter_of<NT>((i * kWaves + wave) * 8 + (lane >> 3), gated), max(n_len - n0, 1) - 1);
    off[4 + i] = (uint32_t)n * (uint32_t)p.w_stride + chunk * 16;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds + wave * 1024;
  // LDS rows of load i: (i * 8 + wave) * 8 ..; an odd tile of 16 is the gated layer's
  const bool odd_tile = gated && (wave >> 1 & 1);
  const char* fb = odd_tile ? ub : wb;

  // One load of step `issued`.  Where the reduction ends inside a row's step, chunks behind its last one are that last
  // one again (inside the row, and zeroed below).
  int issued = 0;
  uint32_t to = 0;
  auto load = [&](int i) {
    load_to_lds_from(i < 4 ? xb : fb, off[i], lds0 + to + i * kWaves * 1024);
  };
  auto begin_step = [&]() {
    if (issued == steps - 1) {
      const int last = (k_len + kChunk - 1) / kChunk - 1;
      const uint32_t back = max(issued * 8 + chunk - last, 0) * 16;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) off[i] -= back;
    }
  };
  auto end_step = [&]() {
    ++issued;
    xb += 128;
    fb += 128;
    to ^= kBuf;
  };
  auto issue = [&]() {
    begin_step();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(i);
    end_step();
  };
  // Step s has landed; zeros behind the reduction's end, in the wave's own part of it.
  auto landed = [&](int s) {
    if (s >= steps) return;
    wait_loads<0>();
    const int valid = k_len - s * kStep - chunk * kChunk;
    if (s == steps - 1 && valid < kChunk) {
      char* mine = lds + (s & 1) * kBuf + wave * 1024 + lane * 16;
#pragma unroll 1
      for (int i = 0; i < kLoads; ++i) {
        uint4* v = reinterpret_cast<uint4*>(mine + i * kWaves * 1024);
        *v = keep_first<TY>(*v, valid);
      }
    }
  };

  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = zero;
  const int wm = wave / 4, wn = wave % 4;
  uint4 a[2][NT], b[2][MT];   // of the two halves of a step
  // LDS addresses of the wave's operands in the two halves of the step that is read next (the kernel's only shared
  // array starts at address 0, its second buffer at bit 16)
  const uint32_t first = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds +
                         (lane & 15) * 128 + ((lane >> 4) ^ (lane >> 1 & 7)) * 16;
  uint32_t xa[2] = {first + wm * MT * 2048, (first ^ 64) + wm * MT * 2048};
  uint32_t wa[2] = {xa[0] + BM * 128 - wm * MT * 2048 + wn * NT * 2048, xa[1] + BM * 128 - wm * MT * 2048 + wn * NT * 2048};
  auto read = [&]() {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < NT; ++j) a[h][j] = read_lds(wa[h] + j * 2048);
#pragma unroll
      for (int i = 0; i < MT; ++i) b[h][i] = read_lds(xa[h] + i * 2048);
      xa[h] ^= kBuf;
      wa[h] ^= kBuf;
    }
  };
  // LOADS: with a load of the coming step between every eight multiplications
  auto multiply = [&](auto loads) {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < MT; ++i) {
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = mfma_chunks<TY>(a[h][j], b[h][i], acc[i][j]);
        if constexpr (decltype(loads)::value) {
          __builtin_amdgcn_sched_barrier(0);
          if (i % 2 == 0) load(h * 4 + i / 2);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    __builtin_amdgcn_s_setprio(0);
  };

  if (steps > 0) {
    issue();
    if (steps > 1) {
      issue();
      wait_loads<kLoads>();
    }
    if (steps == 1) landed(0);
    phase_ends();
    // (as few bodies as there can be without a branch between multiplications: code that runs once costs a fetch from
    // memory every few instructions, 2 us per KB)
    int s = 0;
    if (wave < kWaves / 2) {
      while (s < steps) {
        read();
        if (s >= 1 && issued < steps) issue();
        phase_ends();
        multiply(std::false_type{});
        landed(++s);
        phase_ends();
      }
      phase_ends();
    } else {
      phase_ends();
      for (; s < steps - 2; ++s) {
        read();
        wait_loads<0>();   // step s + 1, not the last
        phase_ends();
        begin_step();
        multiply(std::true_type{});
        end_step();
        phase_ends();
      }
      while (s < steps) {
        read();
        landed(++s);
        phase_ends();
        multiply(std::false_type{});
        phase_ends();
      }
    }
  }
  const int row0 = m0 + wm * MT * 16;
  __syncthreads();   // (no wave reads operands any more)
  constexpr int EM = MT / 2;
  char* mine = lds + wave * EM * 16 * NT * 64;
  if (gated) tile_epilogue<TY, MT, NT, EM, true>(p, acc, mine, e, hi, row0, n0 + wn * NT * 8, n_len, lane);
  else tile_epilogue<TY, MT, NT, EM, false>(p, acc, mine, e, hi, row0, n0 + wn * NT * 16, n_len, lane);
}

}  // namespace

bool linear_wide_applies(const LinearParams& p, fupr_dtype dt) {
  // offsets of 32 bits from the tile's first row (gathered rows: from the first of all) and filter
  const int64_t limit = int64_t(1) << 32;
  return dt != FUPR_F32 && (p.src ? p.x_rows : BM) * p.x_stride <= limit && BN * p.w_stride <= limit;
}

fupr_status launch_linear_wide(LinearParams p, fupr_dtype dt, void* stream) {
  hipStream_t st = (hipStream_t)stream;
  unsigned blocks;
  if (!count_tiles(p, BM, BN, &blocks)) return FUPR_ERR_LIMIT;
  if (dt == FUPR_BF16) linear_wide_kernel<FUPR_BF16><<<dim3(blocks), dim3(kWaves * 64), 0, st>>>(p);
  else linear_wide_kernel<FUPR_F16><<<dim3(blocks), dim3(kWaves * 64), 0, st>>>(p);
  return launch_status("linear_wide_kernel");
}

}  // namespace fupr
