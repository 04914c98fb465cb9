// Products of bf16 matrices on v_mfma_f32_32x32x16_bf16: the tile that the cross entropy of the
// last layer is made of.
//
//   acc[m][n] = sum over pairs (i, j) of sum_k A_i[m][k] B_j[n][k]
//
// An operand lies along k (rows of 16-byte pieces of eight k) or across it (a row for each k), and
// may be several bf16 planes whose sum it is (an fp32 matrix: three); `pairs` lists which planes
// are multiplied with which, and the reduction simply runs over all pairs' k.
//
// Stages of BK k go from memory straight into LDS (16 bytes a lane), into a ring of NBUF
// stages.  Along k, a row's pieces are permuted by its place, so that the sixteen lanes that are
// served together, which read the same piece of sixteen rows, touch all 64 banks (with pieces
// permuted for eight half of the LDS cycles were conflicts).  Across k, fragments are read by
// ds_read_b64_tr_b16 (of sixteen lanes each hands in four m of a k and gets four k of an m),
// and pieces are permuted by k, so that four k by 32 m are 256 different bytes.  Rows beyond
// the operands and k beyond the reduction read as 0.
#pragma once

#include <type_traits>

#include "row_ops.hpp"

namespace luq {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// One operand: planes of [rows][ld] elements; rows and the base are 16-byte aligned.
struct Bf16Planes {
  const uint16_t* p;
  int64_t rows, ld, plane;
};

// Pairs of planes, four bits of each in the order of the reduction.
struct PlanePairs {
  uint32_t a, b;
  int count;
};

struct Bf16Product {
  Bf16Planes A, B;
  PlanePairs pairs;
  int64_t K;           // a multiple of 8 where an operand lies along it
  int tiles_m, tiles_n;
};

// Tile of a workgroup: each XCD takes a run of tiles, eight rows of tiles at a time.
__device__ __forceinline__ void bf16_tile_of(int bid, int ntm, int ntn, int& tm, int& tn) {
  const int total = ntm * ntn, xcd = bid & 7, q = total >> 3, r = total & 7;
  const int at = xcd * q + min(xcd, r) + (bid >> 3);
  constexpr int G = 8;
  const int per = G * ntn, first = (at / per) * G, rows = min(ntm - first, G), in = at - (at / per) * per;
  tm = first + in % rows;
  tn = in / rows;
}

// N fragments that lie across k: of each the reads at address + O1 and + O2, each four k of the lane's
// row.  The wait is in the same block: of a read by the builtin the compiler cannot tell that it does
// not read what the loads to LDS in flight write, and waits for those first (1090 us against 933 for a
// product of 8192 x 4096 over 16000).
typedef short v4h __attribute__((ext_vector_type(4)));
#define LUQ_TR(n, a) "ds_read_b64_tr_b16 %" #n ", %" #a
template <int O1, int O2>
__device__ __forceinline__ void read_across(const uint32_t (&p)[2], v4h (&f)[4]) {
  asm volatile(LUQ_TR(0, 4) " offset:%6\n" LUQ_TR(1, 4) " offset:%7\n"
               LUQ_TR(2, 5) " offset:%6\n" LUQ_TR(3, 5) " offset:%7\n"
               "s_waitcnt lgkmcnt(0)"
               : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
               : "v"(p[0]), "v"(p[1]), "n"(O1), "n"(O2)
               : "memory");
}
template <int O1, int O2>
__device__ __forceinline__ void read_across(const uint32_t (&p)[3], v4h (&f)[6]) {
  asm volatile(LUQ_TR(0, 6) " offset:%9\n" LUQ_TR(1, 6) " offset:%10\n"
               LUQ_TR(2, 7) " offset:%9\n" LUQ_TR(3, 7) " offset:%10\n"
               LUQ_TR(4, 8) " offset:%9\n" LUQ_TR(5, 8) " offset:%10\n"
               "s_waitcnt lgkmcnt(0)"
               : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]), "=&v"(f[5])
               : "v"(p[0]), "v"(p[1]), "v"(p[2]), "n"(O1), "n"(O2)
               : "memory");
}
template <int O1, int O2>
__device__ __forceinline__ void read_across(const uint32_t (&p)[4], v4h (&f)[8]) {
  asm volatile(LUQ_TR(0, 8) " offset:%12\n" LUQ_TR(1, 8) " offset:%13\n"
               LUQ_TR(2, 9) " offset:%12\n" LUQ_TR(3, 9) " offset:%13\n"
               LUQ_TR(4, 10) " offset:%12\n" LUQ_TR(5, 10) " offset:%13\n"
               LUQ_TR(6, 11) " offset:%12\n" LUQ_TR(7, 11) " offset:%13\n"
               "s_waitcnt lgkmcnt(0)"
               : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]), "=&v"(f[5]), "=&v"(f[6]), "=&v"(f[7])
               : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "n"(O1), "n"(O2)
               : "memory");
}
template <int O1, int O2>
__device__ __forceinline__ void read_across(const uint32_t (&p)[6], v4h (&f)[12]) {
  asm volatile(LUQ_TR(0, 12) " offset:%18\n" LUQ_TR(1, 12) " offset:%19\n"
               LUQ_TR(2, 13) " offset:%18\n" LUQ_TR(3, 13) " offset:%19\n"
               LUQ_TR(4, 14) " offset:%18\n" LUQ_TR(5, 14) " offset:%19\n"
               LUQ_TR(6, 15) " offset:%18\n" LUQ_TR(7, 15) " offset:%19\n"
               LUQ_TR(8, 16) " offset:%18\n" LUQ_TR(9, 16) " offset:%19\n"
               LUQ_TR(10, 17) " offset:%18\n" LUQ_TR(11, 17) " offset:%19\n"
               "s_waitcnt lgkmcnt(0)"
               : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]), "=&v"(f[5]), "=&v"(f[6]), "=&v"(f[7]),
                 "=&v"(f[8]), "=&v"(f[9]), "=&v"(f[10]), "=&v"(f[11])
               : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "v"(p[4]), "v"(p[5]), "n"(O1), "n"(O2)
               : "memory");
}
#undef LUQ_TR

template <int WM_, int WN_, int TM_, int TN_, int BK_, int NBUF_>
struct Bf16Tile {
  static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, BK = BK_, NBUF = NBUF_;
  static constexpr int kThreads = 64 * WM * WN, BM = 32 * WM * TM, BN = 32 * WN * TN;
  static constexpr int kRowBytes = BK * 2, kPieces = BK / 8;         // 16-byte pieces of a row
  static constexpr int kStage = (BM + BN) * kRowBytes;
  static constexpr int kLoads = (BM + BN) * kPieces / kThreads;
  static_assert(BM * kPieces % kThreads == 0 && BN * kPieces % kThreads == 0, "whole loads");
  static constexpr int kLds = NBUF * kStage;
  static constexpr int kOut = 0x7FFFFFF0;   // an offset outside every range

  v16f acc[TM][TN];

  // Where a piece of 8 elements lies in an operand's part of a stage: along k [rows][kPieces], across it
  // [BK][edge / 8].
  static __device__ __forceinline__ int along(int row, int piece) {
    return row * kPieces + (piece ^ ((row * kPieces / 16) & (kPieces - 1)));
  }
  template <int EDGE>
  static __device__ __forceinline__ int across(int k, int piece) {
    return k * (EDGE / 8) + (piece ^ ((k & 3) << 2));
  }

  // One operand's view of a stage: its descriptor, and a thread's pieces.
  template <bool CROSS, int EDGE>
  struct Source {
    static constexpr int kCount = EDGE * kPieces / kThreads;
    const Bf16Planes& o;
    int64_t at;          // the tile's first row (along k) or column (across it)
    int ld, span;        // bytes of a row; rows that the tile has
    int off[kCount], k8[kCount];
    __device__ __forceinline__ Source(const Bf16Planes& o_, int64_t at_) : o(o_), at(at_), ld((int)(o_.ld * 2)) {
      span = CROSS ? 0 : (int)min(o.rows - at, (int64_t)EDGE);
#pragma unroll
      for (int i = 0; i < kCount; ++i) {
        const int c = threadIdx.x + i * kThreads;
        if constexpr (CROSS) {
          const int k = c / (EDGE / 8), piece = (c % (EDGE / 8)) ^ ((k & 3) << 2);
          off[i] = k * ld + piece * 16;
          k8[i] = 0;
        } else {
          const int row = c / kPieces, piece = (c % kPieces) ^ ((row * kPieces / 16) & (kPieces - 1));
          off[i] = row * ld + piece * 16;
          k8[i] = piece * 8;
        }
      }
    }
    __device__ __forceinline__ void issue(int plane, int k0, int64_t K, bool live, uint8_t* dst) const {
      const uint16_t* const p = o.p + plane * o.plane + (CROSS ? k0 * o.ld + at : at * o.ld + k0);
      const int bytes = CROSS ? (int)min((int64_t)BK, o.rows - k0) * ld - (int)(at * 2) : span * ld - k0 * 2;
      const auto r = __builtin_amdgcn_make_buffer_rsrc((void*)p, (short)0, live && bytes > 0 ? bytes : 0, 0x00020000);
      const int left = CROSS ? 1 : (int)(K - k0);
#pragma unroll
      for (int i = 0; i < kCount; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(dst + i * kThreads * 16), 16,
                                                 k8[i] < left ? off[i] : kOut, 0, 0, 0);
    }
  };

  // Where in an operand's part of a stage a lane finds its 32-row fragments from row `row0` of the tile on:
  // along k the first piece's row, across it the four m of a k that it hands in.
  static __device__ __forceinline__ int row_of(int row0) { return (row0 + (threadIdx.x & 31)) * kRowBytes; }
  template <int EDGE, int T>
  static __device__ __forceinline__ void columns_of(int row0, int* off) {
    const int lane = threadIdx.x & 63, k = (lane >> 5) * 8 + (lane & 15) / 4, m = row0 + ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
#pragma unroll
    for (int i = 0; i < T; ++i) off[i] = across<EDGE>(k, (m + i * 32) / 8) * 16 + (m & 4) * 2;
  }
  template <int T>
  static __device__ __forceinline__ void read_along(const uint8_t* row, int kk, v8bf (&f)[T]) {
    const int lane = threadIdx.x & 63, swz = ((lane & 31) * kPieces / 16) & (kPieces - 1);
    const int at = ((2 * kk + (lane >> 5)) ^ swz) * 16;
#pragma unroll
    for (int i = 0; i < T; ++i) f[i] = *reinterpret_cast<const v8bf*>(row + i * 32 * kRowBytes + at);
  }
  static __device__ __forceinline__ v8bf join(v4h a, v4h b) {
    return __builtin_bit_cast(v8bf, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }

  // The product of the tile's rows m0.. of A and n0.. of B over stages [beg, end) of the
  // reduction (pairs.count times ceil(K / BK) of them); CA, CB: the operand lies across k.
  template <bool CA, bool CB>
  __device__ __forceinline__ void run(const Bf16Product& g, int64_t m0, int64_t n0, int beg, int end, uint8_t* lds) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int per = (int)((g.K + BK - 1) / BK);
    const Source<CA, BM> from_a(g.A, m0);
    const Source<CB, BN> from_b(g.B, n0);
    // fragments across k: of A first
    constexpr int kCrossA = CA ? TM : 0, kCross = kCrossA + (CB ? TN : 0);
    static_assert((!CA && !CB) || (BM == BN && (CB || !CA)), "B lies across k if A does, of the same edge");
    int off[kCross > 0 ? kCross : 1];
    if constexpr (CA) columns_of<BM, TM>(wm * TM * 32, off);
    if constexpr (CB) columns_of<BN, TN>(wn * TN * 32, off + kCrossA);
    const uint32_t lds_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    const int row_a = row_of(wm * TM * 32), row_b = row_of(wn * TN * 32);
    int pair = beg / per, kt = beg - pair * per;   // of the next stage to be issued
    int issued = beg;
    auto issue = [&](int buf) {
      const bool live = issued < end;
      uint8_t* const dst = lds + buf * kStage + wave * 1024;
      from_a.issue((g.pairs.a >> (4 * pair)) & 15, kt * BK, g.K, live, dst);
      from_b.issue((g.pairs.b >> (4 * pair)) & 15, kt * BK, g.K, live, dst + BM * kRowBytes);
      ++issued;
      if (++kt == per) {
        kt = 0;
        ++pair;
      }
    };
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = v16f{};
    // s_waitcnt immediates (gfx9 encoding): vmcnt alone, lgkmcnt(0) alone
    constexpr int kAhead = (NBUF - 2) * kLoads;
    static_assert(kAhead < 64, "a static wait");
    constexpr int kWaitLoads = (kAhead & 15) | (7 << 4) | (15 << 8) | ((kAhead >> 4) << 14);
    constexpr int kWaitLds = 15 | (7 << 4) | (0 << 8) | (3 << 14);
#pragma unroll
    for (int i = 0; i < NBUF - 1; ++i) issue(i);
    int buf = 0;
    for (int t = beg; t < end; ++t) {
      // own loads of stage t have landed, own reads of stage t - 1 are done; so have everyone's
      __builtin_amdgcn_s_waitcnt(kWaitLds);
      __builtin_amdgcn_s_waitcnt(kWaitLoads);
      asm volatile("s_barrier" ::: "memory");
      const uint8_t* const part_a = lds + buf * kStage;
      const uint8_t* const part_b = part_a + BM * kRowBytes;
      uint32_t at[kCross > 0 ? kCross : 1];
#pragma unroll
      for (int i = 0; i < kCross; ++i)
        at[i] = lds_base + buf * kStage + (i < kCrossA ? 0 : BM * kRowBytes) + off[i];
      auto step = [&](auto constant) {
        constexpr int kk = decltype(constant)::value;
        v8bf a[TM], b[TN];
        if constexpr (!CA) read_along<TM>(part_a + row_a, kk, a);
        if constexpr (!CB) read_along<TN>(part_b + row_b, kk, b);
        if constexpr (kCross > 0) {
          v4h f[2 * kCross];
          constexpr int k0 = kk * 16 * BN * 2;
          read_across<k0, k0 + 4 * BN * 2>(at, f);
#pragma unroll
          for (int i = 0; i < kCrossA; ++i) a[i] = join(f[2 * i], f[2 * i + 1]);
#pragma unroll
          for (int j = 0; j < (CB ? TN : 0); ++j) b[j] = join(f[2 * (kCrossA + j)], f[2 * (kCrossA + j) + 1]);
        }
        // after the first fragments' reads, which the products wait for
        if constexpr (kk == 0) issue(buf == 0 ? NBUF - 1 : buf - 1);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[j], a[i], acc[i][j], 0, 0, 0);
      };
      step(std::integral_constant<int, 0>{});
      step(std::integral_constant<int, 1>{});
      if constexpr (BK == 64) {
        step(std::integral_constant<int, 2>{});
        step(std::integral_constant<int, 3>{});
      }
      buf = buf + 1 == NBUF ? 0 : buf + 1;
    }
    // loads of stages past the end may still be writing into the buffers
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
  }
};

}  // namespace luq
