// Products of bf16 matrices on v_mfma_f32_32x32x16_bf16: the tile that the cross entropy of the
// last layer is made of.
//
//   acc[m][n] = sum over pairs (i, j) of sum_k A_i[m][k] B_j[n][k]
//
// Both operands lie K-major (rows of 16-byte pieces of eight k).  An operand may be several
// bf16 planes whose sum it is (an fp32 matrix: three), and `pairs` lists which planes are
// multiplied with which; the reduction simply runs over all pairs' k.
//
// Stages of kBK k go from memory straight into LDS (16 bytes a lane), rings of NBUF stages: a
// row's pieces are permuted by its place, so that eight lanes that read the same piece of
// eight rows touch all banks.  Rows beyond the operands and k beyond the reduction read as 0.
#pragma once

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
  int64_t K;           // a multiple of 8
  int tiles_m, tiles_n, splits;
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

template <int WM_, int WN_, int TM_, int TN_, int BK_, int NBUF_>
struct Bf16Tile {
  static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, BK = BK_, NBUF = NBUF_;
  static constexpr int kThreads = 64 * WM * WN, BM = 32 * WM * TM, BN = 32 * WN * TN;
  static constexpr int kRowBytes = BK * 2, kPieces = BK / 8;         // 16-byte pieces of a row
  static constexpr int kStage = (BM + BN) * kRowBytes;
  static constexpr int kLoadsA = BM * kPieces / kThreads, kLoads = (BM + BN) * kPieces / kThreads;
  static_assert(BM * kPieces % kThreads == 0 && BN * kPieces % kThreads == 0, "whole loads");
  static constexpr int kLds = NBUF * kStage;
  static constexpr int kOut = 0x7FFFFFF0;   // an offset outside every range

  v16f acc[TM][TN];

  // The product of the tile's rows m0.. of A and n0.. of B over stages [beg, end) of the
  // reduction (pairs.count times ceil(K / BK) of them).
  __device__ __forceinline__ void run(const Bf16Product& g, int64_t m0, int64_t n0, int beg, int end, uint8_t* lds) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int per = (int)((g.K + BK - 1) / BK);
    const int lda = (int)(g.A.ld * 2), ldb = (int)(g.B.ld * 2);
    const int rows_a = (int)min(g.A.rows - m0, (int64_t)BM), rows_b = (int)min(g.B.rows - n0, (int64_t)BN);
    // where a thread's pieces of a stage lie, and which k they begin with
    int src[kLoads], k8[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const bool isb = i >= kLoadsA;
      const int c = tid + (i - (isb ? kLoadsA : 0)) * kThreads, row = c / kPieces, at = c % kPieces;
      const int piece = at ^ ((row * kPieces / 8) & (kPieces - 1));
      src[i] = row * (isb ? ldb : lda) + piece * 16;
      k8[i] = piece * 8;
    }
    int pair = beg / per, kt = beg - pair * per;   // of the next stage to be issued
    int issued = beg;
    auto issue = [&](int buf) {
      const bool live = issued < end;
      const int k0 = kt * BK, left = live ? (int)(g.K - k0) : 0;
      const int pa = (g.pairs.a >> (4 * pair)) & 15, pb = (g.pairs.b >> (4 * pair)) & 15;
      const uint16_t* const a = g.A.p + pa * g.A.plane + m0 * g.A.ld + k0;
      const uint16_t* const b = g.B.p + pb * g.B.plane + n0 * g.B.ld + k0;
      const auto ra = __builtin_amdgcn_make_buffer_rsrc((void*)a, (short)0, live ? rows_a * lda - k0 * 2 : 0, 0x00020000);
      const auto rb = __builtin_amdgcn_make_buffer_rsrc((void*)b, (short)0, live ? rows_b * ldb - k0 * 2 : 0, 0x00020000);
      uint8_t* const dst = lds + buf * kStage + wave * 1024;
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(i < kLoadsA ? ra : rb,
                                                 (__attribute__((address_space(3))) void*)(dst + i * kThreads * 16), 16,
                                                 k8[i] < left ? src[i] : kOut, 0, 0, 0);
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
    const int half = lane >> 5, r = lane & 31;
    int buf = 0;
    for (int t = beg; t < end; ++t) {
      // own loads of stage t have landed, own reads of stage t - 1 are done; so have everyone's
      __builtin_amdgcn_s_waitcnt(kWaitLds);
      __builtin_amdgcn_s_waitcnt(kWaitLoads);
      asm volatile("s_barrier" ::: "memory");
      const uint8_t* const As = lds + buf * kStage + (wm * TM * 32 + r) * kRowBytes;
      const uint8_t* const Bs = lds + buf * kStage + (BM + wn * TN * 32 + r) * kRowBytes;
      const int swz = (r * kPieces / 8) & (kPieces - 1);
#pragma unroll
      for (int kk = 0; kk < BK / 16; ++kk) {
        const int at = ((2 * kk + half) ^ swz) * 16;
        v8bf a[TM], b[TN];
#pragma unroll
        for (int i = 0; i < TM; ++i) a[i] = *reinterpret_cast<const v8bf*>(As + i * 32 * kRowBytes + at);
#pragma unroll
        for (int j = 0; j < TN; ++j) b[j] = *reinterpret_cast<const v8bf*>(Bs + j * 32 * kRowBytes + at);
        // after the first fragments' reads, which the products wait for
        if (kk == 0) issue(buf == 0 ? NBUF - 1 : buf - 1);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[j], a[i], acc[i][j], 0, 0, 0);
      }
      buf = buf + 1 == NBUF ? 0 : buf + 1;
    }
    // loads of stages past the end may still be writing into the buffers
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
  }
};

}  // namespace luq
