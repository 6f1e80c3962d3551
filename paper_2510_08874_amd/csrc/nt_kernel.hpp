// Products of two operands that both lie along K (gfx950, device code only): D[m][n] = sum over k of
// A[m][k] B[n][k], in macro-tiles that one workgroup of four waves accumulates in registers.  Shared by the
// products of 4-bit microscaled operands (mx_kernel.hpp) and of fp16 pairs (ortho_kernel.hpp): both feed a matrix
// instruction with 32 bytes of K a row, 16 in each half of the lanes, so a step, its stage in LDS and its loads are the same:
//   fp4    32 x 32 x 64: a lane holds 32 codes of one row, which share one scale; a step is 256 codes of a row
//   pairs  32 x 32 x 16: a lane holds 8 values of one row; a step is 32 values as high parts (64 bytes) and low parts, whose
//          three products (low high, high low, high high) use what is in LDS three times for two reads
//
// What bounds a 256 x 256 tile: a step of 128 bytes a row is 64 (pairs: 96) matrix instructions of 32 cycles on each of the four
// matrix pipes (2048 cycles, pairs half as many again), 128 KB of LDS reads (1024 cycles at 128 bytes), and 64 KB that loads bring into LDS, which take
// 1950 cycles by themselves (33 bytes a cycle and CU with all CUs at it; 17 TB/s from L2).  L2 answers requests of up to 128
// bytes, so the rows of a step are whole lines.  (With steps of 64 bytes, and four bytes of scales a row
// and step, there were four times as many requests: 16384 x 8192 x 28672 in 4 bits 2.42 ms, matrix pipes busy 35 %.)
// So matrix instructions, LDS reads and loads have to run side by side all the time, from one wave on each SIMD, which issues an
// instruction every four to five cycles: operands go straight into LDS stages, and every load, read and addition has its place between two matrix
// instructions.  fp4: all fragments of a step are read in its first half and the quarter before; behind a barrier its stage is filled
// again in the second half, a quarter before another barrier waits for the step behind it, so that loads of two steps overlap.  Pairs,
// with half as much to load a cycle: fragments of a half are read during the half before it, one barrier a step.
// fp4, 4096 x 4096 x 4096: 2600 cycles a step with 187 instructions besides the matrix instructions.  Before, with 350 of them and one barrier in front of the
// last quarter, 2900, of which matrix instructions and LDS reads alone took 2640, matrix instructions alone 2150.  A tile's ends come on top: 6300
// cycles until the first step has landed, 9300 to store 128 KB of bf16, 19000 for 256 KB of fp32 from every CU at the same time (7 TB/s).
// The part lowers its clock under matrix load: a loop of matrix instructions on registers alone makes 6.5 PFLOP/s in fp4
// and 1.8 in fp16 with random operands (9.7 and 2.5 with zeros), and a kernel that also moves operands has less power left for it
// (1.56 GHz in fp4, pipes busy 63 % of the time; 1.52 with pairs, 85 %).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "mx_launch.hpp"

namespace dmm {

typedef int nt_i32x2 __attribute__((ext_vector_type(2)));
typedef int nt_i32x4 __attribute__((ext_vector_type(4)));
typedef int nt_i32x8 __attribute__((ext_vector_type(8)));
typedef float nt_f32x4 __attribute__((ext_vector_type(4)));
typedef float nt_f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 nt_f16x8 __attribute__((ext_vector_type(8)));
typedef const __attribute__((address_space(1))) char *nt_gptr;
typedef __attribute__((address_space(3))) char *nt_lptr;

constexpr int NT_THREADS = 256;
constexpr int NT_ROW = 128;                // bytes of a row in one step
constexpr int NT_CHUNK = 64;               // what a segment's length is given in: 128 codes, 16 pairs

// 16-byte slots of a 128-byte row are exchanged by row, so that 16 lanes that read one slot of 16 rows fall
// into different banks.
__device__ __forceinline__ int nt_swizzle(int row) { return (row >> 1) & 7; }

// (to byte lds + ON)
template <int ON>
__device__ __forceinline__ void nt_load16(nt_gptr base, unsigned lane_off, unsigned lds) {
  asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(lane_off), "s"(base), "s"(lds), "n"(ON) : "memory", "scc");
}
__device__ __forceinline__ void nt_load4(nt_gptr base, unsigned lane_off, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" : : "v"(lane_off), "s"(base), "s"(lds) : "memory");
}
// (16 bytes on from lane_off, which counts for LDS as well; all lanes if `on` is negative, else none)
__device__ __forceinline__ void nt_load16_if(nt_gptr base, unsigned lane_off, unsigned lds, int on) {
  asm volatile("s_sub_u32 m0, %2, 16\n\ts_ashr_i32 exec_lo, %3, 31\n\ts_mov_b32 exec_hi, exec_lo\n\t"
               "global_load_lds_dwordx4 %0, %1 offset:16\n\ts_mov_b64 exec, -1"
               : : "v"(lane_off), "s"(base), "s"(lds), "s"(on) : "memory", "scc");
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

// Where a slice of 64 rows of a finished tile has an element: columns are exchanged eight at a time by row, so that eight rows
// of a column, eight rows apart, lie in different banks (and eight neighbouring columns of a row stay together).
__device__ __forceinline__ int nt_value(int row, int col, int pitch) { return row * pitch + (col ^ (row & 56)); }

// SCALED: 4-bit codes with scales; otherwise pairs of fp16.  TM x TN macro-tile over WM x (4 / WM) waves, NST stages.
template <bool SCALED_, int TM_, int TN_ = TM_, int NST_ = 2, int WM_ = 2>
struct NtShape {
  static constexpr bool SCALED = SCALED_;
  static constexpr int TM = TM_, TN = TN_, NST = NST_, WM = WM_, WN = 4 / WM;
  static constexpr int MI = TM / WM / 32, NI = TN / WN / 32; // 32 x 32 tiles of a wave
  static constexpr int A_BYTES = TM * NT_ROW, B_BYTES = TN * NT_ROW, STAGE = A_BYTES + B_BYTES;
  // scales of two steps together, 16 bytes a row: a request fetches them once.  Units of 64 rows, A's in front of B's
  static constexpr int S_ROW = 16, S_A = (TM + 63) / 64, S_UNITS = SCALED ? S_A + TN / 64 : 0, S_SLOT = S_UNITS * 64 * S_ROW;
  // slots: of the step that is multiplied, of those under way, and of the one behind them; every step may be a segment's last
  static constexpr int SLOTS = NST + 2;
  static constexpr int LDS = NST * STAGE + SLOTS * S_SLOT;
  static constexpr int LA = TM / 32, LB = TN / 32;           // 1 KB loads of a wave and step, 8 rows each
  static constexpr int LOADS = LA + LB;
  static constexpr int EARLY = LOADS / 2;                    // so many in the third quarter of a step, the others in the last
  static constexpr int LS = (S_UNITS + 3) / 4;               // units of a wave: one with the first of two steps, one with the second
  static_assert(TM % (32 * WM) == 0 && TN % (32 * WN) == 0 && TN % 64 == 0 && LS <= 2, "whole matrix tiles and units of scales");
  static_assert(NST >= 2 && (NST - 1) * LOADS < 64 && LDS <= 160 * 1024, "the counter of loads, the LDS of a CU");
};

// Rows of a macro-tile past `ext` are read from its last row: they are never stored.
template <class SH>
struct NtTile {
  // [i][j][x]: row 32 i + 8 (x / 4) + 4 (lane / 32) + x % 4, column 32 j + lane % 32 of the wave's part
  nt_f32x16 acc[SH::MI][SH::NI];

  // The sums are in accumulator registers here: keeps the compiler from moving them about, and from moving matrix
  // instructions behind a branch.
  __device__ __forceinline__ void pin() {
    nt_for<SH::MI * SH::NI>([&](auto tc) { asm volatile("" : "+a"(acc[decltype(tc)::value / SH::NI][decltype(tc)::value % SH::NI])); });
  }

  // The finished tile, 64 rows at a time through LDS, where `use(values, row)` finds rows row .. row + 31 of the tile in rows 0 .. 31
  // of `values` and row + TM / 2 ... in rows 32 .. 63, every element at nt_value(row, column, PITCH).  Every thread gets there between
  // two barriers.
  static constexpr int PITCH = SH::TN + 4;
  template <class F>
  __device__ __forceinline__ void slices(char *lds, F &&use) {
    static_assert(SH::WM == 2 && 64 * PITCH * 4 <= SH::LDS, "a slice is 64 rows and lies in the stages");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float *const values = (float *)lds;
    float *const mine = values + ((wave >> 1) * 32 + 4 * (lane >> 5)) * PITCH;
    const int col = (wave & 1) * (SH::TN / 2) + (lane & 31), turn = (wave >> 1) * 32;
    nt_for<SH::MI>([&](auto ic) {
      constexpr int I = decltype(ic)::value;
      __syncthreads();
      nt_for<SH::NI>([&](auto jc) {
        constexpr int J = decltype(jc)::value;
#pragma unroll
        for (int x = 0; x < 16; ++x) mine[(8 * (x / 4) + x % 4) * PITCH + ((col + 32 * J) ^ (turn + x / 4 * 8))] = acc[I][J][x];
        __builtin_amdgcn_sched_barrier(0);
      });
      __syncthreads();
      use(values, 32 * I);
    });
  }

  // `front`: the segment that holds the first step, step `first` of it; `segs`: n_segs from that one on (read from the second
  // on); `steps`: in all, one at least.  A segment of an odd number of chunks ends with half a step.
  __device__ __forceinline__ void run(const NtSeg &front, const NtSeg *segs, int n_segs, int first, int steps, int m_off, int m_ext, int n_off, int n_ext,
                                      char *lds) {
    constexpr int MI = SH::MI, NI = SH::NI, LA = SH::LA, LB = SH::LB;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / SH::WN, wn = wave % SH::WN;
    const unsigned lds0 = (unsigned)(uintptr_t)(nt_lptr)lds;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = nt_f32x16{};

    // ---- this lane's part of the loads -----------------------------------------------------
    // load x of a wave: rows 8 (4 x + wave) ..., 16 bytes a lane, in the order of the stage
    const int row8 = 8 * wave + (lane >> 3);
    const int slot = (lane & 7) ^ nt_swizzle(row8);          // (load x is 32 rows on: the same)
    unsigned aoff[LA], boff[LB];
    nt_gptr a = nullptr, b = nullptr;
    int chunks = 0, on = NT_ROW;                              // chunks left to load in this segment; bytes from one step to the next
    // scales: this wave's units, at sp those of row 0 of the unit's operand and the segment's next two steps
    const bool s_is_a[2] = {wave < SH::S_A, wave + 4 < SH::S_A};
    const int s_row[2] = {64 * (s_is_a[0] ? wave : wave - SH::S_A), 64 * (s_is_a[1] ? wave + 4 : wave + 4 - SH::S_A)};
    const int s_ext[2] = {(s_is_a[0] ? m_ext : n_ext) - 1, (s_is_a[1] ? m_ext : n_ext) - 1};
    nt_gptr sp[2] = {nullptr, nullptr};
    unsigned s_pitch[2] = {0, 0}, soff[2] = {0, 0};
    bool s_wide = false;                                      // 16 bytes of a row at a time
    auto enter = [&](const NtSeg &s, int skip) {
      chunks = s.chunks - 2 * skip;
      a = nt_uniform(s.a + (int64_t)m_off * s.a_pitch + (int64_t)skip * NT_ROW);
      b = nt_uniform(s.b + (int64_t)n_off * s.b_pitch + (int64_t)skip * NT_ROW);
#pragma unroll
      for (int x = 0; x < LA; ++x) aoff[x] = __umul24(min(32 * x + row8, m_ext - 1), s.a_pitch) + slot * 16;
#pragma unroll
      for (int x = 0; x < LB; ++x) boff[x] = __umul24(min(32 * x + row8, n_ext - 1), s.b_pitch) + slot * 16;
      if constexpr (SH::SCALED) {
        s_wide = true;
#pragma unroll
        for (int x = 0; x < SH::LS; ++x) {
          s_pitch[x] = s_is_a[x] ? s.a_scale_pitch : s.b_scale_pitch;
          sp[x] = nt_uniform((s_is_a[x] ? s.a_scale : s.b_scale) + (int64_t)(s_is_a[x] ? m_off : n_off) * s_pitch[x] + (int64_t)skip * 8);
          s_wide = s_wide && (((unsigned)(uintptr_t)sp[x] | s_pitch[x]) & 15) == 0;
          soff[x] = __umul24(min(s_row[x] + lane, s_ext[x]), s_pitch[x]);
        }
      }
    };
    // The step that is loaded next is half a one: the lanes of what is missing read the half that is there, and count for nothing, since
    // their scales are 2^-127 on both sides (fp16 operands are filled up with zeros).
    auto halve = [&]() {
      if (chunks == 1) {
        const unsigned back = slot >= 4 ? 64 : 0;
#pragma unroll
        for (int x = 0; x < LA; ++x) aoff[x] -= back;
#pragma unroll
        for (int x = 0; x < LB; ++x) boff[x] -= back;
      }
    };
    // load x of a step, into the stage at byte `base` of LDS
    auto load = [&](auto xc, unsigned base) {
      constexpr int X = decltype(xc)::value;
      if constexpr (X < LA) nt_load16<X * 4096>(a, aoff[X], base + wave * 1024);
      else nt_load16<SH::A_BYTES + (X - LA) * 4096>(b, boff[X - LA], base + wave * 1024);
    };
    // Scales of two steps at a time, in the next slot.
    int s_left = 0;                                           // steps that the slot has scales of and that are yet to be loaded
    unsigned s_at = 0, s_slot = (SH::SLOTS - 1) * SH::S_SLOT; // where those of the step loaded next are; the slot filled last
    unsigned s_loaded[SH::NST - 1] = {};                      // ... of the last NST - 1 steps loaded, in their order
    auto s_behind = [&]() { return s_slot == (SH::SLOTS - 1) * SH::S_SLOT ? 0 : s_slot + SH::S_SLOT; };
    // Of the two steps that follow, at once and word by word: in front of a segment, at its end, and where scales lie at
    // odd places.  What is missing is 2^-127.
    auto load_scales = [&]() {
      if constexpr (SH::SCALED) {
        const int n = chunks < 4 ? chunks : 4;
        const unsigned d = lane & 3;
#pragma unroll
        for (int y = 0; y < SH::LS; ++y) {
          if (wave + 4 * y >= SH::S_UNITS) break;
          const unsigned to = SH::NST * SH::STAGE + s_slot + (wave + 4 * y) * (64 * SH::S_ROW);
          if (n == 4 && s_wide) {
            nt_load16<0>(sp[y], soff[y], lds0 + to);
          } else if (n == 4) {
#pragma unroll
            for (int x = 0; x < 4; ++x) nt_load4(sp[y], __umul24(min(s_row[y] + 16 * x + (lane >> 2), s_ext[y]), s_pitch[y]) + d * 4, lds0 + to + x * 256);
          } else {
            for (int x = 0; x < 4; ++x) {
              int v = 0;
              if ((int)d < n)
                v = *(const __attribute__((address_space(1))) int *)(sp[y] + (__umul24(min(s_row[y] + 16 * x + (lane >> 2), s_ext[y]), s_pitch[y]) + d * 4));
              *(__attribute__((address_space(3))) int *)((nt_lptr)lds + to + x * 256 + lane * 4) = v;
            }
          }
        }
      }
    };
    auto new_slot = [&]() {
      s_slot = s_behind();
      s_at = s_slot;
      s_left = chunks > 2 ? 2 : 1;
    };
    // Elsewhere those of the next two steps are loaded during these two, a unit of a wave with each.  s_rest: chunks behind the steps
    // of the slot, where 16 bytes of a row can be loaded at a time; little or nothing: word by word.
    int s_rest = 0;
    const unsigned s_mine = lds0 + SH::NST * SH::STAGE + wave * (64 * SH::S_ROW);
    auto count_rest = [&]() { s_rest = s_wide ? chunks - 2 * s_left : 0; };
    auto load_scales_ahead = [&]() {
      if constexpr (SH::SCALED) {
        const int left = s_left;
        const bool second = SH::LS > 1 && left == 1;
        int on = 3 - s_rest;
        if constexpr (SH::S_UNITS < 4 * SH::LS) on = wave + (left == 1 ? 4 : 0) < SH::S_UNITS ? on : 0;
        if constexpr (SH::LS == 1) on = left == 1 ? 0 : on;
        nt_load16_if(second ? sp[1] : sp[0], second ? soff[1] : soff[0], s_mine + s_behind() + (second ? 4 * 64 * SH::S_ROW : 0), on);
      }
    };
    int seg = 0;
    enter(front, first);
    halve();
    new_slot();
    load_scales();
    count_rest();
    // To the next step to load, in two parts: what every step needs, which runs between matrix instructions, and the rest, seldom.
    // Past the last step its operands are loaded again, to be read by nobody.
    bool fresh = false;                                       // the next step's scales are the first of a slot
    auto next_scales = [&]() {
      if constexpr (SH::SCALED) {
#pragma unroll
        for (int x = 0; x + 1 < SH::NST - 1; ++x) s_loaded[x] = s_loaded[x + 1];
        s_loaded[SH::NST - 2] = s_at;
        int m = (s_left - 2) >> 31;                           // -1 behind the last step of a slot
        asm("" : "+s"(m));                                    // (selects by one condition would become a branch, and all matrix instructions come behind it)
        fresh = m != 0;
        s_slot = fresh ? s_behind() : s_slot;
        s_at = fresh ? s_slot : s_at + 8;
        s_left += (m & 2) - 1;
        s_rest += m & -4;
#pragma unroll
        for (int x = 0; x < SH::LS; ++x) sp[x] += m & 16;
      }
    };
    auto next_operands = [&]() {
      a += on;
      b += on;
      chunks -= 2;
    };
    auto next_rest = [&]() {
      if (chunks <= 2 || (SH::SCALED && fresh && (!s_wide || chunks < 4))) {
        if (chunks <= 0) {
          if (++seg < n_segs) {
            enter(segs[seg], 0);
            halve();
            if (!fresh) s_slot = s_behind();
            s_at = s_slot;
            s_left = chunks > 2 ? 2 : 1;
            load_scales();
            count_rest();
          } else {
            a -= on;
            b -= on;
            on = 0;
            chunks = s_left = 1 << 30;
            s_rest = 0;
          }
        } else {
          halve();
          if (SH::SCALED && fresh) {
            s_left = chunks > 2 ? 2 : 1;
            load_scales();
          }
        }
      }
    };
    auto next = [&]() {
      next_scales();
      next_operands();
      next_rest();
    };

    // ---- fragments ---------------------------------------------------------------------------
    // quarter h of a step: 32 bytes of 32 rows, 16 in each lane.  A row's scales (8 bytes a step) are shifted once so that byte
    // 2 (h % 2) of word h / 2 is the one of the lane's codes.
    const int r = lane & 31, g = lane >> 5;
    const nt_lptr fa = (nt_lptr)lds + wm * (SH::TM / SH::WM) * NT_ROW + r * NT_ROW;
    const nt_lptr fb = (nt_lptr)lds + SH::A_BYTES + wn * (SH::TN / SH::WN) * NT_ROW + r * NT_ROW;
    const nt_lptr fs = (nt_lptr)lds + SH::NST * SH::STAGE + r * SH::S_ROW;
    const int turn = (g ^ nt_swizzle(r)) * 16;                // (slot 2 h + g, exchanged)
    struct Frag {
      nt_i32x4 a[MI], b[NI];
    };
    struct Scale {                                            // [word of a row's eight bytes][rows of A, columns of B]
      int v[2][SH::SCALED ? MI + NI : 1];
    };
    // fragment x of a quarter: the rows of A, the columns of B
    auto read = [&](Frag &f, auto xc, unsigned stage, auto hc) {
      constexpr int X = decltype(xc)::value;
      const unsigned o = stage + (turn ^ (decltype(hc)::value * 32));
      if constexpr (X < MI) f.a[X] = *(const __attribute__((address_space(3))) nt_i32x4 *)(fa + o + X * 32 * NT_ROW);
      else f.b[X - MI] = *(const __attribute__((address_space(3))) nt_i32x4 *)(fb + o + (X - MI) * 32 * NT_ROW);
    };
    // both words of a row as they are (one by one they keep LDS busy for 400 cycles more a step)
    struct RawScale {
      nt_i32x2 v[SH::SCALED ? MI + NI : 1];
    };
    auto read_scale = [&](RawScale &f, auto xc, unsigned at) {
      if constexpr (SH::SCALED) {
        constexpr int X = decltype(xc)::value;
        const nt_lptr p = fs + at;
        if constexpr (X < MI) f.v[X] = *(const __attribute__((address_space(3))) nt_i32x2 *)(p + (wm * (SH::TM / SH::WM) + 32 * X) * SH::S_ROW);
        else f.v[X] = *(const __attribute__((address_space(3))) nt_i32x2 *)(p + (64 * SH::S_A + wn * (SH::TN / SH::WN) + 32 * (X - MI)) * SH::S_ROW);
      }
    };
    // word W for the lane's half
    auto shift = [&](Scale &f, const RawScale &raw, auto xc, auto wc) {
      if constexpr (SH::SCALED) {
        int &v = f.v[decltype(wc)::value][decltype(xc)::value];
        v = (int)((unsigned)raw.v[decltype(xc)::value][decltype(wc)::value] >> (8 * g));
        asm volatile("" : "+v"(v));                           // here, not in front of its use
      }
    };
    auto multiply = [&](const Frag &f, const Scale &s, auto tc, auto hc) {
      if constexpr (SH::SCALED) {
        constexpr int H = decltype(hc)::value, I = decltype(tc)::value / NI, J = decltype(tc)::value % NI;
        const nt_i32x8 x = {f.a[I][0], f.a[I][1], f.a[I][2], f.a[I][3], 0, 0, 0, 0};
        const nt_i32x8 y = {f.b[J][0], f.b[J][1], f.b[J][2], f.b[J][3], 0, 0, 0, 0};
        acc[I][J] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, acc[I][J], 4, 4, 2 * (H & 1), s.v[H >> 1][I], 2 * (H & 1), s.v[H >> 1][MI + J]);
      }
    };
    // of pairs: a's part times b's (0: high, 1: low)
    struct Pair {
      Frag part[SH::SCALED ? 1 : 2];
    };
    auto multiply_pair = [&](const Pair &f, auto tc, auto ac, auto bc) {
      if constexpr (!SH::SCALED) {
        constexpr int I = decltype(tc)::value / NI, J = decltype(tc)::value % NI;
        acc[I][J] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(nt_f16x8, f.part[decltype(ac)::value].a[I]),
                                                           __builtin_bit_cast(nt_f16x8, f.part[decltype(bc)::value].b[J]), acc[I][J], 0, 0, 0);
      }
    };
    constexpr int T = MI * NI, R = MI + NI;
    // The order of the statements is the order of the instructions: what else a quarter needs (its `also`, by matrix instruction)
    // is spread over its matrix instructions, which take the pipe 32 cycles each.
    auto quarter = [&](const Frag &f, const Scale &s, auto hc, auto also) {
      nt_for<T>([&](auto tc) {
        multiply(f, s, tc, hc);
        also(tc);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    // calls f with those of 0 ... N - 1 that belong to matrix instruction `tc`, if they are spread over the first L of them
    auto spread = [&](auto nc, auto lc, auto tc, auto f) {
      constexpr int N = decltype(nc)::value, L = decltype(lc)::value;
      nt_for<N>([&](auto xc) {
        if constexpr (decltype(xc)::value * L / N == decltype(tc)::value) f(xc);
      });
    };
    // Half h of a step of pairs (values 16 h ...): the small products first.  Reads half 1 - h of `stage` into `into`.
    auto half = [&](const Pair &f, auto hc, Pair &into, unsigned stage, auto also) {
      constexpr int H = decltype(hc)::value;
      nt_for<3 * T>([&](auto tc) {
        constexpr int I = decltype(tc)::value;
        multiply_pair(f, std::integral_constant<int, I % T>{}, std::integral_constant<int, I < T>{}, std::integral_constant<int, I / T == 1>{});
        nt_for<2 * R>([&](auto xc) {
          constexpr int X = decltype(xc)::value;
          // (in the order of their use: low parts of A, high ones of B, ...)
          if constexpr (X * 3 * T / (2 * R) == I) read(into.part[X < R ? (X < MI) : (X - R >= MI)], std::integral_constant<int, X % R>{}, stage,
                                                       std::integral_constant<int, 1 - H + 2 * (X < R ? (X < MI) : (X - R >= MI))>{});
        });
        also(tc);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    std::integral_constant<int, 0> h0;
    std::integral_constant<int, 1> h1;
    std::integral_constant<int, 2> h2;
    std::integral_constant<int, 3> h3;
    auto nothing = [](auto) {};

    // ---- the steps ---------------------------------------------------------------------------
    // in front: all stages under way, the first fragments of step 0 read
    unsigned s_first = 0;
#pragma unroll
    for (int x = 0; x < SH::NST; ++x) {
      nt_for<SH::LOADS>([&](auto xc) { load(xc, lds0 + x * SH::STAGE); });
      load_scales_ahead();
      next();
      if (x == 0) s_first = s_loaded[SH::NST - 2];
    }
    nt_wait_loads<(SH::NST - 1) * SH::LOADS>();               // (and the step's scales, older or behind a wait of their own)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    unsigned now = 0;                                         // stage of the current step
    if constexpr (SH::SCALED) {
      // A wave issues an instruction every four or five cycles, so no more than six between two matrix instructions; what a barrier or
      // the next quarter waits for is issued a few of these ahead.
      constexpr int R2 = R * 3 / 4;
      constexpr std::integral_constant<int, T> all;
      constexpr std::integral_constant<int, (T * 11 + 15) / 16> most;
      constexpr std::integral_constant<int, R> n_frags;
      Frag f0, f1, f2, f3;
      Scale s;
      RawScale raw;
      nt_for<R>([&](auto xc) { read_scale(raw, xc, s_first); });
      nt_for<R>([&](auto xc) { shift(s, raw, xc, h0); });
      nt_for<R>([&](auto xc) { read(f0, xc, 0, h0); });
#pragma clang loop unroll(disable)
      do {
        const unsigned behind = now == (SH::NST - 1) * SH::STAGE ? 0 : now + SH::STAGE;
        unsigned s_next = 0;
        // All of this step's fragments are read in three quarters: its stage may be filled a quarter before the next one
        // has to have landed.
        quarter(f0, s, h0, [&](auto tc) {
          spread(std::integral_constant<int, R + R2>{}, all, tc, [&](auto xc) {
            constexpr int X = decltype(xc)::value;
            if constexpr (X < R) read(f1, xc, now, h1);
            else read(f2, std::integral_constant<int, X - R>{}, now, h2);
          });
          spread(n_frags, all, tc, [&](auto xc) { shift(s, raw, xc, h1); });
          if constexpr (decltype(tc)::value == T / 8) load_scales_ahead();
        });
        quarter(f1, s, h1, [&](auto tc) {
          spread(std::integral_constant<int, 2 * R - R2>{}, most, tc, [&](auto xc) {
            constexpr int X = decltype(xc)::value + R2;
            if constexpr (X < R) read(f2, std::integral_constant<int, X>{}, now, h2);
            else read(f3, std::integral_constant<int, X - R>{}, now, h3);
          });
          if constexpr (decltype(tc)::value == T * 12 / 16) {
            s_next = s_loaded[0];                             // where the next step's are
            next_scales();
          }
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // every wave has read them
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        quarter(f2, s, h2, [&](auto tc) {
          spread(std::integral_constant<int, SH::EARLY>{}, all, tc, [&](auto xc) { load(xc, lds0 + now); });
        });
        nt_wait_loads<(SH::NST - 2) * SH::LOADS + SH::EARLY>();   // the next step has landed
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        quarter(f3, s, h3, [&](auto tc) {
          constexpr int X = decltype(tc)::value;
          spread(std::integral_constant<int, SH::LOADS - SH::EARLY>{}, most, tc, [&](auto xc) { load(std::integral_constant<int, decltype(xc)::value + SH::EARLY>{}, lds0 + now); });
          spread(n_frags, most, tc, [&](auto xc) { read_scale(raw, xc, s_next); });
          spread(n_frags, most, tc, [&](auto xc) { read(f0, xc, behind, h0); });
          if constexpr (X == T * 13 / 16) next_operands();
          nt_for<R>([&](auto xc) {
            if constexpr (T * 12 / 16 + decltype(xc)::value * (T - T * 12 / 16) / R == X) shift(s, raw, xc, h0);
          });
        });
        pin();
        next_rest();
        now = behind;
      } while (--steps > 0);
    } else {
      Pair f0, f1;
      nt_for<R>([&](auto xc) {
        read(f0.part[1], xc, 0, h2);
        read(f0.part[0], xc, 0, h0);
      });
#pragma clang loop unroll(disable)
      do {
        const unsigned behind = now == (SH::NST - 1) * SH::STAGE ? 0 : now + SH::STAGE;
        half(f0, h0, f1, now, nothing);
        nt_wait_loads<(SH::NST - 2) * SH::LOADS>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        half(f1, h1, f0, behind, [&](auto tc) {               // ... and the loads of the step that gets this one's stage
          nt_for<SH::LOADS>([&](auto xc) {
            if constexpr (decltype(xc)::value * 3 * T / SH::LOADS == decltype(tc)::value) load(xc, lds0 + now);
          });
        });
        now = behind;
        pin();
        next();
      } while (--steps > 0);
    }
    nt_wait_loads<0>();
  }
};

}  // namespace dmm
