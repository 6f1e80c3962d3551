// Macro-tiles of the products around a layer (gfx950, device code only): D[m][n] = sum over k of A[m][k] B[k][n] of 8-bit
// integers or bf16, which one workgroup of four waves accumulates in registers.
//
// Both feed a matrix instruction of 32 x 32 results with 32 bytes of K a row, 16 in each half of the lanes (i8: 32 of K, bf16: 16), and
// both take the pipe 32 cycles, so that a step, its stage in LDS and its loads are the same whatever the elements:
//   direct operand (along K in memory)    a step is 128 bytes of every row; fragments are read 16 bytes at a time
//   turned operand (across K; bf16 alone) a step is 64 rows of 128 columns at a time; fragments come from transposing reads, which
//                                         give a lane four k of its column
// A gated product has two right operands: the stage holds 128 columns of each, and a wave multiplies 32 columns of one and the same 32 of the
// other in turn, so that both sums of an element end in one lane, where the activation needs them.
//
// What bounds a 256 x 256 tile: a step is 64 matrix instructions on each of four pipes (2048 cycles), 128 KB of LDS reads (1024) and
// 64 KB that loads bring into LDS (1950 with all CUs at it), which have to run side by side from one wave on each SIMD.  As in the
// products of 4-bit operands, all fragments of a step are read in its first half and the quarter before; behind a barrier its stage is
// filled again in the second half, a quarter before another barrier waits for the step behind it.
//
// Measured, whole products: integers 2.41 to 2.56 POP/s (16384 x 8192 x 28672), bf16 1.30 to 1.36 PFLOP/s gated (8192 x 12288 x 49152), 1.40
// along K and across K (both gradients of 8192^3), where the library's largest product makes 1.41 and the pipes alone 1.77 to 1.81 from registers.  A step takes
// 1.37 to 1.42 us of which matrix instructions are 1.19, a tile's ends (first stages, epilogue) 8 to 11 us of 64 steps' 90.
//
// Shapes, and what each is for:
//   256 x 256         one workgroup a CU, 256 accumulators a lane: the most work for a byte of LDS
//   128 x 128         two on a CU (gated: 128 x (64 + 64) in integers, 64 x (128 + 128) in bf16): where 256 x 256 would leave CUs idle, and one's ends run
//                     beside the other's steps (8-bit gated 256 x 2048 x 2048 11.4 us, one 128 x (128 + 128) a CU 17.2)
//   64 x 128, 32 x 128   few rows; what bounds them is B's way from memory, so stages are as many as LDS holds: where every workgroup has a CU to itself 6
//                     and 7 of them (one row, 8192 x 28672 in 8 bits from memory: 48 to 54 us, 54 with three stages; 43 at the 5.5 TB/s of a large read)
//
// K of any length and rows at any address: whole steps of all segments come first, then what is left of each segment, 16 bytes at a time, moved to the front
// where the row ends and filled up with zeros.  Such a tail takes about 5 us (loads that everything waits for), which is what the copies of finely cut
// operands save.
#pragma once

#include "layer_launch.hpp"
#include "nt_kernel.hpp"

namespace dmm {

typedef __bf16 layer_bf16x8 __attribute__((ext_vector_type(8)));
typedef short layer_i16x4 __attribute__((ext_vector_type(4)));
typedef int layer_i32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) layer_i16x4 *layer_lds_i16x4;

constexpr int LAYER_THREADS = 256;
constexpr int LAYER_SUB = 128;             // columns of a turned operand that lie together in a stage
constexpr int LAYER_SUB_BYTES = 64 * 256;  // 64 k rows of them

// TM x TN macro-tile (of a gated product: TN / 2 columns of each right operand) over WM x (4 / WM) waves, NST stages.
template <int KIND_, int TM_, int TN_, int NST_, int WM_>
struct LayerShape {
  static constexpr int KIND = KIND_, TM = TM_, TN = TN_, NST = NST_, WM = WM_, WN = 4 / WM;
  static constexpr bool I8 = layer_i8(KIND), DUAL = layer_gated(KIND), A_TURNED = KIND == LAYER_TN, B_TURNED = KIND == LAYER_TN || KIND == LAYER_GATED;
  static constexpr int ES = I8 ? 1 : 2, STEP = 128 / ES, CHUNK = 16 / ES;   // elements of a step, of 16 bytes
  static constexpr int MI = TM / WM / 32, NI = TN / WN / 32;  // 32 x 32 tiles of a wave
  static constexpr int OUT = DUAL ? TN / 2 : TN;              // columns of the result
  static constexpr int A_BYTES = TM * 128, B_BYTES = TN * 128, STAGE = A_BYTES + B_BYTES, LDS = NST * STAGE;
  static constexpr int LA = TM / 32, LB = TN / 32, LOADS = LA + LB;   // 1 KB loads of a wave and step
  static constexpr int EARLY = LOADS / 2;                     // so many in the third quarter of a step, the others in the last
  static_assert(TM % (32 * WM) == 0 && TN % (32 * WN) == 0 && (!DUAL || NI % 2 == 0), "whole matrix tiles");
  static_assert((!A_TURNED || TM % LAYER_SUB == 0) && (!B_TURNED || TN % LAYER_SUB == 0) && (!DUAL || !B_TURNED || TN == 2 * LAYER_SUB), "whole blocks of columns");
  static_assert(NST >= 2 && (NST - 1) * LOADS < 64 && LDS <= 160 * 1024, "the counter of loads, the LDS of a CU");
};

// `n` elements (at most 16 bytes' worth) at p, zeros behind them.  Where the row has 16 bytes up to there (`before` elements in front of p) these are read and
// moved to the front: one by one, a row's end kept every wave waiting up to 15 times.
template <int ES>
__device__ __forceinline__ nt_i32x4 layer_some(const char *p, int n, int before) {
  nt_i32x4 v = {0, 0, 0, 0};
  if (n >= 16 / ES) {
    __builtin_memcpy(&v, p, 16);
  } else if (n > 0 && before + n >= 16 / ES) {
    unsigned __int128 all;
    const int back = 16 - n * ES;
    __builtin_memcpy(&all, p - back, 16);
    v = __builtin_bit_cast(nt_i32x4, all >> (8 * back));
  } else if (n > 0) {
    unsigned w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16 / ES; ++i)
      if (i < n) {
        const unsigned e = ES == 1 ? (unsigned)*(const unsigned char *)(p + i) : ES == 2 ? (unsigned)*(const unsigned short *)(p + 2 * i) : *(const unsigned *)(p + 4 * i);
        w[i * ES / 4] |= e << (i * ES % 4 * 8);
      }
    v = nt_i32x4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
  }
  return v;
}

// Rows (columns) of a macro-tile past `ext` hold something that is never stored.
template <class SH>
struct LayerTileSums {
  using Acc = std::conditional_t<SH::I8, layer_i32x16, nt_f32x16>;
  // [i][j][x]: row 32 i + 8 (x / 4) + 4 (lane / 32) + x % 4, column 32 j + lane % 32 of the wave's part; gated: column 32 (j / 2) + lane % 32
  // of right operand j % 2
  Acc acc[SH::MI][SH::NI];

  // The sums are in accumulator registers here: keeps the compiler from moving them about, and from moving matrix
  // instructions behind a branch.
  __device__ __forceinline__ void pin() {
    nt_for<SH::MI * SH::NI>([&](auto tc) { asm volatile("" : "+a"(acc[decltype(tc)::value / SH::NI][decltype(tc)::value % SH::NI])); });
  }

  // `segs`: it.n_segs from it.seg on (read from the second on), `tails`: those whose tails it adds.
  __device__ __forceinline__ void run(const LayerItem &it, const LayerSeg *segs, const LayerSeg *tails, char *lds) {
    constexpr int MI = SH::MI, NI = SH::NI, LA = SH::LA, LB = SH::LB;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / SH::WN, wn = wave % SH::WN;
    const unsigned lds0 = (unsigned)(uintptr_t)(nt_lptr)lds;
    const int m_off = it.m_off, m_ext = it.m_ext, n_off = it.n_off, n_ext = it.n_ext;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = Acc{};

    // ---- fragments ---------------------------------------------------------------------------
    // quarter h of a step: 32 bytes of K of 32 rows, 16 in each lane
    const int r = lane & 31, g = lane >> 5;
    const int turn = (g ^ nt_swizzle(r)) * 16;                // direct: slot 2 h + g of a row, exchanged by row
    // turned: in each group of 16 lanes, lane i names 4 columns of k row i / 4 and receives column i of those 4 rows.  64-byte pieces of
    // a k row are exchanged by k, so that the four rows lie in different banks
    const int gr = lane >> 4, li = lane & 15;
    const int t_row = ((gr >> 1) * 8 + (li >> 2)) * 256 + ((gr & 1) * 2 + ((li & 3) >> 1)) * 16 + (li & 1) * 8, t_turn = li >> 2;
    int fa[SH::A_TURNED ? MI : 1], fb[SH::B_TURNED ? NI : 1];
    if constexpr (SH::A_TURNED) {
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int t = wm * MI + i;
        fa[i] = (t >> 2) * LAYER_SUB_BYTES + t_row + ((t & 3) ^ t_turn) * 64;
      }
    } else {
      fa[0] = (wm * (SH::TM / SH::WM) + r) * 128;
    }
    if constexpr (SH::B_TURNED) {
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int t = SH::DUAL ? (j & 1) * 4 + wn * (NI / 2) + j / 2 : wn * NI + j;
        fb[j] = SH::A_BYTES + (t >> 2) * LAYER_SUB_BYTES + t_row + ((t & 3) ^ t_turn) * 64;
      }
    } else {
      fb[0] = SH::A_BYTES + (wn * (SH::OUT / SH::WN) + r) * 128;
    }
    struct Frag {
      nt_i32x4 a[MI], b[NI];
    };
    auto turned = [&](int at, auto hc) {
      union {
        layer_i16x4 h[2];
        nt_i32x4 v;
      } u;
      u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((layer_lds_i16x4)((nt_lptr)lds + at + (16 * decltype(hc)::value) * 256));
      u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((layer_lds_i16x4)((nt_lptr)lds + at + (16 * decltype(hc)::value + 4) * 256));
      return u.v;
    };
    // fragment x of a quarter: the rows of A, the columns of B
    auto read = [&](Frag &f, auto xc, unsigned stage, auto hc) {
      constexpr int X = decltype(xc)::value, H = decltype(hc)::value;
      if constexpr (X < MI) {
        if constexpr (SH::A_TURNED) f.a[X] = turned(fa[X] + (int)stage, hc);
        else f.a[X] = *(const __attribute__((address_space(3))) nt_i32x4 *)((nt_lptr)lds + fa[0] + (stage + (turn ^ (H * 32))) + X * 32 * 128);
      } else {
        constexpr int J = X - MI;
        if constexpr (SH::B_TURNED) f.b[J] = turned(fb[J] + (int)stage, hc);
        else f.b[J] = *(const __attribute__((address_space(3))) nt_i32x4 *)((nt_lptr)lds + fb[0] + (stage + (turn ^ (H * 32))) +
                                                                            (SH::DUAL ? (J & 1) * SH::OUT + J / 2 * 32 : J * 32) * 128);
      }
    };
    auto multiply = [&](const Frag &f, auto tc) {
      constexpr int I = decltype(tc)::value / NI, J = decltype(tc)::value % NI;
      if constexpr (SH::I8) acc[I][J] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.a[I], f.b[J], acc[I][J], 0, 0, 0);
      else acc[I][J] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(layer_bf16x8, f.a[I]), __builtin_bit_cast(layer_bf16x8, f.b[J]),
                                                               acc[I][J], 0, 0, 0);
    };
    constexpr int T = MI * NI, R = MI + NI;
    std::integral_constant<int, 0> h0;
    std::integral_constant<int, 1> h1;
    std::integral_constant<int, 2> h2;
    std::integral_constant<int, 3> h3;

    int steps = it.steps;
    if (steps > 0) {
      // ---- this lane's part of the loads -----------------------------------------------------
      // direct, load x of a wave: rows 8 (4 x + wave) ..., 16 bytes a lane, in the order of the stage
      const int row8 = 8 * wave + (lane >> 3);
      const int slot = (lane & 7) ^ nt_swizzle(row8);         // (load x is 32 rows on: the same)
      // turned: k rows 4 (4 (x % 4) + wave) ... of block x / 4
      const int k4 = 4 * wave + gr, chunk = ((((lane & 15) >> 2) ^ (gr & 3)) << 2) | (lane & 3);
      unsigned aoff[LA], boff[LB];
      nt_gptr a = nullptr, b = nullptr, b2 = nullptr;
      int left = 0;                                           // whole steps left to load in this segment
      int on_a = 0, on_b = 0, on_b2 = 0;                      // bytes from one step to the next
      auto enter = [&](const LayerSeg &s, int skip) {
        left = s.steps - skip;
        on_a = SH::A_TURNED ? __builtin_amdgcn_readfirstlane((int)(64 * s.a_pitch)) : 128;
        on_b = SH::B_TURNED ? __builtin_amdgcn_readfirstlane((int)(64 * s.b_pitch)) : 128;
        a = nt_uniform(s.a + (SH::A_TURNED ? (int64_t)m_off * SH::ES : (int64_t)m_off * s.a_pitch) + (int64_t)skip * on_a);
        b = nt_uniform(s.b + (SH::B_TURNED ? (int64_t)n_off * SH::ES : (int64_t)n_off * s.b_pitch) + (int64_t)skip * on_b);
        if constexpr (SH::DUAL) {
          on_b2 = SH::B_TURNED ? __builtin_amdgcn_readfirstlane((int)(64 * s.b2_pitch)) : 128;
          b2 = nt_uniform(s.b2 + (SH::B_TURNED ? (int64_t)n_off * SH::ES : (int64_t)n_off * s.b2_pitch) + (int64_t)skip * on_b2);
        }
#pragma unroll
        for (int x = 0; x < LA; ++x) {
          if constexpr (SH::A_TURNED) aoff[x] = __umul24(16 * (x % 4) + k4, s.a_pitch) + min(x / 4 * 16 + chunk, (m_ext - 1) >> 3) * 16;
          else aoff[x] = __umul24(min(32 * x + row8, m_ext - 1), s.a_pitch) + slot * 16;
        }
#pragma unroll
        for (int x = 0; x < LB; ++x) {
          constexpr int HALF = SH::DUAL ? LB / 2 : LB;
          const uint32_t pitch = SH::DUAL && x >= HALF ? s.b2_pitch : s.b_pitch;
          if constexpr (SH::B_TURNED) boff[x] = __umul24(16 * (x % 4) + k4, pitch) + min(x % HALF / 4 * 16 + chunk, (n_ext - 1) >> 3) * 16;
          else boff[x] = __umul24(min(32 * (x % HALF) + row8, n_ext - 1), pitch) + slot * 16;
        }
      };
      auto load = [&](auto xc, unsigned base) {
        constexpr int X = decltype(xc)::value;
        if constexpr (X < LA) nt_load16<X * 4096>(a, aoff[X], base + wave * 1024);
        else if constexpr (SH::DUAL && X - LA >= LB / 2) nt_load16<SH::A_BYTES + (X - LA) * 4096>(b2, boff[X - LA], base + wave * 1024);
        else nt_load16<SH::A_BYTES + (X - LA) * 4096>(b, boff[X - LA], base + wave * 1024);
      };
      int seg = 0;
      enter(it.front, it.first);
      // To the next step to load.  Past the last step its operands are loaded again, to be read by nobody.
      auto next_operands = [&]() {
        a += on_a;
        b += on_b;
        if constexpr (SH::DUAL) b2 += on_b2;
        --left;
      };
      auto next_rest = [&]() {
        if (left > 0) return;
        do ++seg;
        while (seg < it.n_segs && segs[seg].steps == 0);
        if (seg < it.n_segs) {
          enter(segs[seg], 0);
        } else {
          a -= on_a;
          b -= on_b;
          if constexpr (SH::DUAL) b2 -= on_b2;
          on_a = on_b = on_b2 = 0;
          left = 1 << 30;
        }
      };
      // The order of the statements is the order of the instructions: what else a quarter needs (its `also`, by matrix instruction)
      // is spread over its matrix instructions, which take the pipe 32 cycles each.
      auto quarter = [&](const Frag &f, auto also) {
        nt_for<T>([&](auto tc) {
          multiply(f, tc);
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
      // in front: all stages under way, the first fragments of step 0 read
#pragma unroll
      for (int x = 0; x < SH::NST; ++x) {
        nt_for<SH::LOADS>([&](auto xc) { load(xc, lds0 + x * SH::STAGE); });
        next_operands();
        next_rest();
      }
      nt_wait_loads<(SH::NST - 1) * SH::LOADS>();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      unsigned now = 0;                                       // stage of the current step
      constexpr int R2 = R * 3 / 4;
      constexpr std::integral_constant<int, T> all;
      constexpr std::integral_constant<int, (T * 11 + 15) / 16> most;
      constexpr std::integral_constant<int, R> n_frags;
      Frag f0, f1, f2, f3;
      nt_for<R>([&](auto xc) { read(f0, xc, 0, h0); });
#pragma clang loop unroll(disable)
      do {
        const unsigned behind = now == (SH::NST - 1) * SH::STAGE ? 0 : now + SH::STAGE;
        quarter(f0, [&](auto tc) {
          spread(std::integral_constant<int, R + R2>{}, all, tc, [&](auto xc) {
            constexpr int X = decltype(xc)::value;
            if constexpr (X < R) read(f1, xc, now, h1);
            else read(f2, std::integral_constant<int, X - R>{}, now, h2);
          });
        });
        quarter(f1, [&](auto tc) {
          spread(std::integral_constant<int, 2 * R - R2>{}, most, tc, [&](auto xc) {
            constexpr int X = decltype(xc)::value + R2;
            if constexpr (X < R) read(f2, std::integral_constant<int, X>{}, now, h2);
            else read(f3, std::integral_constant<int, X - R>{}, now, h3);
          });
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // every wave has read them
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        quarter(f2, [&](auto tc) {
          spread(std::integral_constant<int, SH::EARLY>{}, all, tc, [&](auto xc) { load(xc, lds0 + now); });
        });
        nt_wait_loads<(SH::NST - 2) * SH::LOADS + SH::EARLY>();   // the next step has landed
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        quarter(f3, [&](auto tc) {
          spread(std::integral_constant<int, SH::LOADS - SH::EARLY>{}, most, tc,
                 [&](auto xc) { load(std::integral_constant<int, decltype(xc)::value + SH::EARLY>{}, lds0 + now); });
          spread(n_frags, most, tc, [&](auto xc) { read(f0, xc, behind, h0); });
          if constexpr (decltype(tc)::value == T * 13 / 16) next_operands();
        });
        pin();
        next_rest();
        now = behind;
      } while (--steps > 0);
      nt_wait_loads<0>();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }

    // ---- what whole steps leave of the segments, in stage 0 -------------------------------------
    for (int x = 0; x < it.n_tails; ++x) {
      const LayerSeg s = tails[x];
      if (s.tail == 0) continue;
      // 16 bytes a thread and y, of A or of B, and where they belong
      auto some = [&](bool of_b, int y) {
        const bool second = SH::DUAL && of_b && y >= LB / 2, is_turned = of_b ? SH::B_TURNED : SH::A_TURNED;
        const char *const p = of_b ? (second ? s.b2 : s.b) : s.a;
        const int64_t pitch = of_b ? (second ? s.b2_pitch : s.b_pitch) : s.a_pitch;
        const int off = of_b ? n_off : m_off, ext = of_b ? n_ext : m_ext, at = (second ? y - LB / 2 : y) * 256 + tid;
        if (is_turned) {
          const int k = at >> 4 & 63, col = (at >> 10) * LAYER_SUB + (at & 15) * 8;
          return layer_some<SH::ES>(p + (int64_t)(off + col) * SH::ES + ((int64_t)s.steps * 64 + k) * pitch, k < s.tail ? ext - col : 0, off + col);
        }
        const int row = at >> 3, k = (at & 7) * SH::CHUNK;
        return layer_some<SH::ES>(p + (int64_t)(off + row) * pitch + ((int64_t)s.steps * SH::STEP + k) * SH::ES, row < ext ? s.tail - k : 0,
                                  s.steps > 0 ? SH::CHUNK : k);
      };
      auto keep = [&](bool of_b, int y, nt_i32x4 v) {
        const int at = y * 256 + tid;
        int to = of_b ? SH::A_BYTES : 0;
        if (of_b ? SH::B_TURNED : SH::A_TURNED) {
          const int k = at >> 4 & 63, c = at & 15;
          to += (at >> 10) * LAYER_SUB_BYTES + k * 256 + (((c >> 2) ^ (k & 3)) << 2 | (c & 3)) * 16;
        } else {
          const int row = at >> 3;
          to += row * 128 + ((at & 7) ^ nt_swizzle(row)) * 16;
        }
        *(__attribute__((address_space(3))) nt_i32x4 *)((nt_lptr)lds + to) = v;
      };
      __syncthreads();                                        // every wave is done with the stage
      // (four at a time beside 256 accumulators a lane, else all of them: each time is a wait for memory)
      constexpr int MOST = MI * NI <= 4 ? SH::LOADS : 4;
#pragma unroll
      for (int y0 = 0; y0 < SH::LOADS; y0 += MOST) {
        nt_i32x4 v[MOST];
#pragma unroll
        for (int y = 0; y < MOST; ++y)
          if (y0 + y < SH::LOADS) v[y] = y0 + y < LA ? some(false, y0 + y) : some(true, y0 + y - LA);
#pragma unroll
        for (int y = 0; y < MOST; ++y)
          if (y0 + y < SH::LOADS) y0 + y < LA ? keep(false, y0 + y, v[y]) : keep(true, y0 + y - LA, v[y]);
        __builtin_amdgcn_sched_barrier(0);
      }
      __syncthreads();
      const int quarters = (s.tail * SH::ES + 31) / 32;
      nt_for<4>([&](auto hc) {
        if (decltype(hc)::value < quarters) {
          Frag f;
          nt_for<R>([&](auto xc) { read(f, xc, 0, hc); });
          nt_for<T>([&](auto tc) { multiply(f, tc); });
        }
        pin();
      });
    }
  }
};

}  // namespace dmm
