// Products of two operands that both lie along K (gfx950, device code only): D[m][n] = sum over k of
// A[m][k] B[n][k], in macro-tiles that one workgroup of four waves accumulates in registers.  Shared by the
// products of 4-bit microscaled operands (mx_kernel.hpp) and of fp16 pairs (ortho_kernel.hpp): both feed a matrix
// instruction with 64 bytes of K a row, 16 in each lane, so a step, its stage in LDS and its loads are the same:
//   fp4   16 x 16 x 128: a lane holds 32 codes of one row, which share one scale
//   fp16  16 x 16 x 32:  a lane holds 8 values of one row
//
// What bounds a 256 x 256 tile: a step is 64 matrix instructions of 16 cycles on each of the four matrix
// pipes (1024 cycles), 64 KB of LDS reads (512 cycles at 128 bytes), 32 KB written to LDS by the loads (256) and 32
// KB from L2 (32 bytes a cycle and CU).  So the pipes can be kept busy if nothing waits: operands go straight into
// a ring of four LDS stages, two steps ahead, and the fragments of a step are read during the step before it,
// between its matrix instructions.  One barrier a step: behind it the next step's stage may be read, and the stage of
// the step before, which every wave has read, may be filled.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "mx_launch.hpp"

namespace dmm {

typedef int nt_i32x4 __attribute__((ext_vector_type(4)));
typedef int nt_i32x8 __attribute__((ext_vector_type(8)));
typedef float nt_f32x4 __attribute__((ext_vector_type(4)));
typedef float nt_f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 nt_f16x8 __attribute__((ext_vector_type(8)));
typedef const __attribute__((address_space(1))) char *nt_gptr;
typedef __attribute__((address_space(3))) char *nt_lptr;

constexpr int NT_THREADS = 256;
constexpr int NT_ROW = 64;                 // bytes of a row in one step
constexpr int NT_STAGES = 4;

// 16-byte slots of a 64-byte row are exchanged by row, so that 16 lanes that read one slot of 16 rows fall
// into different banks.
__device__ __forceinline__ int nt_swizzle(int row) { return ((row >> 1) & 3) ^ ((row >> 3) & 1); }

__device__ __forceinline__ void nt_load16(nt_gptr base, unsigned lane_off, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(lane_off), "s"(base), "s"(lds) : "memory");
}
__device__ __forceinline__ void nt_load4(nt_gptr base, unsigned lane_off, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" : : "v"(lane_off), "s"(base), "s"(lds) : "memory");
}
template <int N>
__device__ __forceinline__ void nt_wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ nt_gptr nt_uniform(const char *p) {
  const uint64_t v = (uint64_t)p;
  return (nt_gptr)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}

template <int N, class F, int... I>
__device__ __forceinline__ void nt_for_impl(std::integer_sequence<int, I...>, F &&f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void nt_for(F &&f) {
  nt_for_impl<N>(std::make_integer_sequence<int, N>{}, f);
}

// SCALED: 4-bit codes with scales; otherwise fp16.  TM x TN macro-tile over 2 x 2 waves.
template <bool SCALED_, int TM_, int TN_>
struct NtShape {
  static constexpr bool SCALED = SCALED_;
  static constexpr int TM = TM_, TN = TN_;
  static constexpr int MI = TM / 64, NI = TN / 64;           // 32 x 32 tiles of a wave
  static constexpr int A_BYTES = TM * NT_ROW, B_BYTES = TN * NT_ROW;
  static constexpr int S_BYTES = SCALED ? (TM + TN) * 4 : 0;
  static constexpr int STAGE = A_BYTES + B_BYTES + S_BYTES;
  static constexpr int LDS = NT_STAGES * STAGE;
  static constexpr int LA = TM / 64, LB = TN / 64;           // 1 KB loads of a wave and step
  static constexpr int LS = SCALED ? (TM + TN) / 256 : 0;    // 64-row loads of scales of a wave and step
  static constexpr int LOADS = LA + LB + LS;
  static_assert(TM % 128 == 0 && TN % 128 == 0, "a wave loads whole rows of scales");
};

// Rows of a macro-tile past `ext` are read from its last row: they are never stored.
template <class SH>
struct NtTile {
  // [i][j][x]: row 32 i + 8 (x / 4) + 4 (lane / 32) + x % 4, column 32 j + lane % 32 of the wave's quarter
  nt_f32x16 acc[SH::MI][SH::NI];

  // The sums are in accumulator registers here: keeps the compiler from moving them about.
  __device__ __forceinline__ void pin() {
    nt_for<SH::MI * SH::NI>([&](auto tc) { asm volatile("" : "+a"(acc[decltype(tc)::value / SH::NI][decltype(tc)::value % SH::NI])); });
  }

  // `segs`: n_segs from the one that holds the first step; `first`: the first step in it; `steps`: in all
  // The finished tile, 64 rows at a time through LDS, where `use(values, row)` finds rows row .. row + 31 of the tile in rows 0 .. 31
  // of `values` and row + TM / 2 ... in rows 32 .. 63; PITCH floats from one to the next.  Every thread gets there between two barriers.
  static constexpr int PITCH = SH::TN + 4;
  static_assert(64 * PITCH * 4 <= SH::LDS, "a slice lies in the stages");
  template <class F>
  __device__ __forceinline__ void slices(char *lds, F &&use) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float *const values = (float *)lds;
    float *const mine = values + ((wave >> 1) * 32 + 4 * (lane >> 5)) * PITCH + (wave & 1) * (SH::TN / 2) + (lane & 31);
    nt_for<SH::MI>([&](auto ic) {
      constexpr int I = decltype(ic)::value;
      __syncthreads();
      nt_for<SH::NI>([&](auto jc) {
        constexpr int J = decltype(jc)::value;
#pragma unroll
        for (int x = 0; x < 16; ++x) mine[(8 * (x / 4) + x % 4) * PITCH + 32 * J] = acc[I][J][x];
        __builtin_amdgcn_sched_barrier(0);
      });
      __syncthreads();
      use(values, 32 * I);
    });
  }

  // (`segs`: anything that has an NtSeg at an index)
  template <class Segs>
  __device__ __forceinline__ void run(const Segs &segs, int n_segs, int first, int steps, int m_off, int m_ext, int n_off, int n_ext, char *lds) {
    constexpr int MI = SH::MI, NI = SH::NI, LA = SH::LA, LB = SH::LB, LS = SH::LS;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const unsigned lds0 = (unsigned)(uintptr_t)(nt_lptr)lds;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = nt_f32x16{};
    if (steps <= 0) return;

    // ---- this lane's part of the loads -----------------------------------------------------
    // load x of a wave: rows 16 (4 x + wave) ..., 16 bytes a lane, in the order of the stage
    int arow[LA], brow[LB], srow[LS ? LS : 1];
#pragma unroll
    for (int x = 0; x < LA; ++x) arow[x] = min(16 * (4 * x + wave) + (lane >> 2), m_ext - 1);
#pragma unroll
    for (int x = 0; x < LB; ++x) brow[x] = min(16 * (4 * x + wave) + (lane >> 2), n_ext - 1);
    // load x of scales: rows 64 (LS wave + x) ... of A's rows followed by B's
#pragma unroll
    for (int x = 0; x < LS; ++x) {
      const int row = 64 * (LS * wave + x) + lane;
      srow[x] = 64 * (LS * wave + x) < SH::TM ? min(row, m_ext - 1) : min(row - SH::TM, n_ext - 1);
    }
    const int slot = ((lane & 3) ^ nt_swizzle(lane >> 2)) * 16;
    unsigned aoff[LA], boff[LB], soff[LS ? LS : 1];
    nt_gptr a = nullptr, b = nullptr, as = nullptr, bs = nullptr;
    int left = 0, on = NT_ROW;                                // steps to load in this run of K; bytes from one to the next
    auto enter = [&](const NtSeg &s, int skip) {
      left = s.steps - skip;
      a = nt_uniform(s.a + (int64_t)m_off * s.a_pitch + (int64_t)skip * NT_ROW);
      b = nt_uniform(s.b + (int64_t)n_off * s.b_pitch + (int64_t)skip * NT_ROW);
#pragma unroll
      for (int x = 0; x < LA; ++x) aoff[x] = (unsigned)arow[x] * s.a_pitch + slot;
#pragma unroll
      for (int x = 0; x < LB; ++x) boff[x] = (unsigned)brow[x] * s.b_pitch + slot;
      if constexpr (SH::SCALED) {
        as = nt_uniform(s.a_scale + (int64_t)m_off * s.a_scale_pitch + (int64_t)skip * 4);
        bs = nt_uniform(s.b_scale + (int64_t)n_off * s.b_scale_pitch + (int64_t)skip * 4);
#pragma unroll
        for (int x = 0; x < LS; ++x) soff[x] = (unsigned)srow[x] * (64 * (LS * wave + x) < SH::TM ? s.a_scale_pitch : s.b_scale_pitch);
      }
    };
    int seg = 0;
    enter(segs[0], first);
    // load x of a step, into the stage at byte `base` of LDS
    auto load = [&](auto xc, unsigned base) {
      constexpr int X = decltype(xc)::value;
      if constexpr (X < LA) nt_load16(a, aoff[X], base + (4 * X + wave) * 1024);
      else if constexpr (X < LA + LB) nt_load16(b, boff[X - LA], base + SH::A_BYTES + (4 * (X - LA) + wave) * 1024);
      else {
        constexpr int Y = X - LA - LB;
        nt_load4(64 * (LS * wave + Y) < SH::TM ? as : bs, soff[Y], base + SH::A_BYTES + SH::B_BYTES + (LS * wave + Y) * 256);
      }
    };
    // to the next step to load.  Past the last one its operands are loaded again, to be read by nobody: the loads under
    // way stay countable, and the loop has no branches
    auto advance = [&]() {
      a += on;
      b += on;
      if constexpr (SH::SCALED) {
        as += on >> 4;
        bs += on >> 4;
      }
    };
    auto turn = [&]() {                                       // behind the last step of a run
      if (seg + 1 < n_segs) {
        ++seg;
        enter(segs[seg], 0);
      } else {
        a -= on;
        b -= on;
        as -= on >> 4;
        bs -= on >> 4;
        on = 0;
        left = 1 << 30;
      }
    };

    // ---- fragments ---------------------------------------------------------------------------
    // half h of a step: 32 bytes of 32 rows, 16 in each lane; a row's scales (4 bytes a step) are shifted once so
    // that byte 2 h is the one of the lane's codes
    const int r = lane & 31, g = lane >> 5;
    const nt_lptr fa = (nt_lptr)lds + wm * (SH::TM / 2) * NT_ROW + r * NT_ROW;
    const nt_lptr fb = (nt_lptr)lds + SH::A_BYTES + wn * (SH::TN / 2) * NT_ROW + r * NT_ROW;
    const nt_lptr fs = (nt_lptr)lds + SH::A_BYTES + SH::B_BYTES + r * 4;
    const int chunk[2] = {(g ^ nt_swizzle(r)) * 16, ((2 + g) ^ nt_swizzle(r)) * 16};
    struct Frag {
      nt_i32x4 a[MI], b[NI];
    };
    struct Scale {
      int a[SH::SCALED ? MI : 1], b[SH::SCALED ? NI : 1];
    };
    // fragment x of a half: the rows of A, the columns of B
    auto read = [&](Frag &f, auto xc, unsigned stage, auto hc) {
      constexpr int X = decltype(xc)::value;
      const unsigned o = stage + chunk[decltype(hc)::value];
      if constexpr (X < MI) f.a[X] = *(const __attribute__((address_space(3))) nt_i32x4 *)(fa + o + X * 32 * NT_ROW);
      else f.b[X - MI] = *(const __attribute__((address_space(3))) nt_i32x4 *)(fb + o + (X - MI) * 32 * NT_ROW);
    };
    auto read_scales = [&](Scale &f, unsigned stage) {
      if constexpr (SH::SCALED) {
        const nt_lptr p = fs + stage;
#pragma unroll
        for (int i = 0; i < MI; ++i) f.a[i] = *(const __attribute__((address_space(3))) int *)(p + (wm * (SH::TM / 2) + 32 * i) * 4);
#pragma unroll
        for (int j = 0; j < NI; ++j) f.b[j] = *(const __attribute__((address_space(3))) int *)(p + (SH::TM + wn * (SH::TN / 2) + 32 * j) * 4);
      }
    };
    auto shift = [&](Scale &f) {
      if constexpr (SH::SCALED) {
#pragma unroll
        for (int i = 0; i < MI; ++i) f.a[i] = (int)((unsigned)f.a[i] >> (8 * g));
#pragma unroll
        for (int j = 0; j < NI; ++j) f.b[j] = (int)((unsigned)f.b[j] >> (8 * g));
      }
    };
    auto multiply = [&](const Frag &f, const Scale &s, auto tc, auto hc) {
      constexpr int H = decltype(hc)::value, I = decltype(tc)::value / NI, J = decltype(tc)::value % NI;
      if constexpr (SH::SCALED) {
        const nt_i32x8 x = {f.a[I][0], f.a[I][1], f.a[I][2], f.a[I][3], 0, 0, 0, 0};
        const nt_i32x8 y = {f.b[J][0], f.b[J][1], f.b[J][2], f.b[J][3], 0, 0, 0, 0};
        acc[I][J] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, acc[I][J], 4, 4, 2 * H, s.a[I], 2 * H, s.b[J]);
      } else {
        acc[I][J] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(nt_f16x8, f.a[I]), __builtin_bit_cast(nt_f16x8, f.b[J]), acc[I][J], 0, 0, 0);
      }
    };
    std::integral_constant<int, 0> h0;
    std::integral_constant<int, 1> h1;
    constexpr int T = MI * NI, R = MI + NI;

    // ---- the steps ---------------------------------------------------------------------------
    // in front: stages 0, 1 and 2 under way, the first half of step 0 read
#pragma unroll
    for (int x = 0; x < 3; ++x) {
      nt_for<SH::LOADS>([&](auto xc) { load(xc, lds0 + x * SH::STAGE); });
      advance();
      if (--left == 0) turn();
    }
    nt_wait_loads<2 * SH::LOADS>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    Frag f0, f1;
    Scale s, s_next;
    read_scales(s, 0);
    nt_for<R>([&](auto xc) { read(f0, xc, 0, h0); });
    unsigned now = 0, fill = 3 * SH::STAGE;                   // stage of the current step; stage that is filled next
    // The order of the statements is the order of the instructions: what else a step needs is spread over its
    // matrix instructions, which take the pipe 32 cycles each.
#pragma clang loop unroll(disable)
    for (int t = steps; t > 0; --t) {
      shift(s);
      nt_for<T>([&](auto tc) {
        constexpr int I = decltype(tc)::value;
        multiply(f0, s, tc, h0);
        nt_for<R>([&](auto xc) {
          if constexpr (decltype(xc)::value * T / R == I) read(f1, xc, now, h1);
        });
        __builtin_amdgcn_sched_barrier(0);
      });
      nt_wait_loads<SH::LOADS>();                           // the next step has landed
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      now = now == 3 * SH::STAGE ? 0 : now + SH::STAGE;
      const unsigned base = lds0 + fill;
      fill = fill == 3 * SH::STAGE ? 0 : fill + SH::STAGE;
      read_scales(s_next, now);
      __builtin_amdgcn_sched_barrier(0);
      nt_for<T>([&](auto tc) {
        constexpr int I = decltype(tc)::value;
        multiply(f1, s, tc, h1);
        nt_for<R>([&](auto xc) {
          if constexpr (decltype(xc)::value * T / R == I) read(f0, xc, now, h0);
        });
        nt_for<SH::LOADS>([&](auto xc) {
          if constexpr (decltype(xc)::value * T / SH::LOADS == I) load(xc, base);
        });
        __builtin_amdgcn_sched_barrier(0);
      });
      advance();
      s = s_next;
      pin();                                                  // (or the compiler moves matrix instructions behind the branch)
      if (--left == 0) turn();
    }
    nt_wait_loads<0>();
  }
};

}  // namespace dmm
