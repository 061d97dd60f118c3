// What the products of two 4-bit matrices share: the tiles of a step, how they lie in a stage, and the block-scaled instructions
// (tcgen05.mma kind::mxf4 / mxf4nvf4) that multiply them.
#pragma once

#include "pvt_mma.cuh"
#include "pvt_mx.cuh"

#ifdef __CUDACC__
namespace pvt {
namespace mx {
namespace {

constexpr int kTileW = 128;      // rows of w
constexpr int kRowBytes = 128;   // of a step
constexpr uint32_t kFewTokens = 16;

// of the kernel for few tokens
template <int FMT>
struct FewSizes {
  static constexpr uint32_t KT = FMT == PVT_MX_E8M0_32 ? 2 : 4;  // scale tiles of a step and strip
  // a stage: rows of w, rows of x, scales of w, scales of x
  static constexpr uint32_t kX = kTileW * kRowBytes, kWs = kX + kFewTokens * kRowBytes, kXs = kWs + KT * kTileBytes;
  static constexpr uint32_t kStage = kXs + KT * kTileBytes, kStageAligned = (kStage + 1023) / 1024 * 1024;
  static constexpr uint32_t kStages = 110 * 1024 / kStageAligned;  // of two blocks per SM
  static constexpr uint32_t kScaleCols = KT * 4 * 2;
  static constexpr uint32_t kTmem = 32 + kStages * kScaleCols <= 128 ? 128 : 256;
  static_assert(32 + kStages * kScaleCols <= kTmem, "sums and scales fit");
  static constexpr size_t kBytes = kStages * kStageAligned + 1024;
  static_assert(kFewTokens * kTileW * 4 <= kStages * kStageAligned, "the partial sums fit the stages");
};

__device__ __forceinline__ void scales_to_tmem(uint32_t taddr, uint64_t desc) {
  asm volatile(
      "{\n\t.reg .pred one;\n\t"
      "elect.sync _|one, 0xffffffff;\n\t"
      "@one tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(taddr), "l"(desc)
      : "memory");
}
// 64 columns of all rows of a tile
template <int FMT>
__device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                         uint32_t onto) {
  if (FMT == PVT_MX_E8M0_32) {
    asm volatile(
        "{\n\t.reg .pred one, p;\n\t"
        "elect.sync _|one, 0xffffffff;\n\t"
        "setp.ne.u32 p, %6, 0;\n\t"
        "@one tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(onto)
        : "memory");
  } else {
    asm volatile(
        "{\n\t.reg .pred one, p;\n\t"
        "elect.sync _|one, 0xffffffff;\n\t"
        "setp.ne.u32 p, %6, 0;\n\t"
        "@one tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(onto)
        : "memory");
  }
}

// ---- pairs of blocks ----
constexpr int kPairReaders = 8;  // warps
constexpr int kPairCopyWarps = 2;  // (a warp takes 100 cycles and more for each copy it issues)
constexpr int kPairCopyWarp = kPairReaders, kPairMmaWarp = kPairCopyWarp + kPairCopyWarps;
constexpr int kPairThreads = (kPairMmaWarp + 1) * 32;
constexpr uint32_t kPairRows = 256;   // of w
constexpr uint32_t kPairStages = 7;   // at most
constexpr uint32_t kLeastSteps = 12;  // of a pair that shares a tile with others

// N: rows of x in a tile
template <int FMT, uint32_t N>
struct PairSizes {
  static constexpr uint32_t KT = FMT == PVT_MX_E8M0_32 ? 2 : 4, kStrips = N / kStrip;
  static constexpr uint32_t kX = kTileW * kRowBytes, kWs = kX + N / 2 * kRowBytes, kXs = kWs + KT * kTileBytes;
  static constexpr uint32_t kStage = kXs + kStrips * KT * kTileBytes, kStageAligned = (kStage + 1023) / 1024 * 1024;
  static constexpr uint32_t kScaleCols = KT * 4 * (1 + kStrips);  // of a stage
  static constexpr uint32_t kStages = N == 256 ? 5 : 7;
  static_assert(N + kStages * kScaleCols <= 512, "sums and scales fit tensor memory");
  static constexpr size_t kBytes = kStages * kStageAligned + 1024;
  static_assert(kBytes + 1024 <= 227 * 1024 && kStages <= kPairStages, "a block's shared memory");
  static_assert(N * kTileW * 4 <= kStages * kStageAligned, "the partial sums fit the stages");
};

// A step of a pair: its scales to tensor memory (two or four tiles for w's 128 rows, as many for each of one or two strips of
// x) and the products of four times 64 columns.  One thread is elected for all of them, and descriptors are counted on inside:
// a tile of scales is 32 units of 16 bytes, four columns of tensor memory; 64 columns are 2 units of either operand.
template <int FMT, uint32_t STRIPS>
__device__ __forceinline__ void multiply_step(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                              uint64_t w_scales, uint64_t x_scales, uint32_t onto) {
  if constexpr (FMT == PVT_MX_E8M0_32 && STRIPS == 2) {
    asm volatile(
        "{\n\t"
        ".reg .pred one, p, t;\n\t"
        ".reg .b32 s, x, i;\n\t"
        ".reg .b64 q, a, b;\n\t"
        "elect.sync _|one, 0xffffffff;\n\t"
        "setp.ne.u32 p, %8, 0;\n\t"
        "setp.eq.u32 t, 0, 0;\n\t"
        "add.u32 s, %4, 0;\n\t"
        "add.s64 q, %6, 0;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [s], q;\n\t"
        "add.u32 x, %5, 0;\n\t"
        "add.s64 q, %7, 0;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 x, %5, 4;\n\t"
        "add.s64 q, %7, 64;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 s, %4, 4;\n\t"
        "add.s64 q, %6, 32;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [s], q;\n\t"
        "add.u32 x, %5, 8;\n\t"
        "add.s64 q, %7, 32;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 x, %5, 12;\n\t"
        "add.s64 q, %7, 96;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.s64 a, %1, 0;\n\t"
        "add.s64 b, %2, 0;\n\t"
        "add.u32 s, %4, 0;\n\t"
        "add.u32 x, %5, 0;\n\t"
        "or.b32 i, %3, 0;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], a, b, i, [s], [x], p;\n\t"
        "add.s64 a, %1, 2;\n\t"
        "add.s64 b, %2, 2;\n\t"
        "add.u32 s, %4, 0;\n\t"
        "add.u32 x, %5, 0;\n\t"
        "or.b32 i, %3, 1073741856;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], a, b, i, [s], [x], t;\n\t"
        "add.s64 a, %1, 4;\n\t"
        "add.s64 b, %2, 4;\n\t"
        "add.u32 s, %4, 4;\n\t"
        "add.u32 x, %5, 8;\n\t"
        "or.b32 i, %3, 0;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], a, b, i, [s], [x], t;\n\t"
        "add.s64 a, %1, 6;\n\t"
        "add.s64 b, %2, 6;\n\t"
        "add.u32 s, %4, 4;\n\t"
        "add.u32 x, %5, 8;\n\t"
        "or.b32 i, %3, 1073741856;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], a, b, i, [s], [x], t;\n\t"
        "}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "l"(w_scales), "l"(x_scales), "r"(onto)
        : "memory");
  } else if constexpr (FMT == PVT_MX_E8M0_32) {
    asm volatile(
        "{\n\t"
        ".reg .pred one, p, t;\n\t"
        ".reg .b32 s, x, i;\n\t"
        ".reg .b64 q, a, b;\n\t"
        "elect.sync _|one, 0xffffffff;\n\t"
        "setp.ne.u32 p, %8, 0;\n\t"
        "setp.eq.u32 t, 0, 0;\n\t"
        "add.u32 s, %4, 0;\n\t"
        "add.s64 q, %6, 0;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [s], q;\n\t"
        "add.u32 x, %5, 0;\n\t"
        "add.s64 q, %7, 0;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 s, %4, 4;\n\t"
        "add.s64 q, %6, 32;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [s], q;\n\t"
        "add.u32 x, %5, 4;\n\t"
        "add.s64 q, %7, 32;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.s64 a, %1, 0;\n\t"
        "add.s64 b, %2, 0;\n\t"
        "add.u32 s, %4, 0;\n\t"
        "add.u32 x, %5, 0;\n\t"
        "or.b32 i, %3, 0;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], a, b, i, [s], [x], p;\n\t"
        "add.s64 a, %1, 2;\n\t"
        "add.s64 b, %2, 2;\n\t"
        "add.u32 s, %4, 0;\n\t"
        "add.u32 x, %5, 0;\n\t"
        "or.b32 i, %3, 1073741856;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], a, b, i, [s], [x], t;\n\t"
        "add.s64 a, %1, 4;\n\t"
        "add.s64 b, %2, 4;\n\t"
        "add.u32 s, %4, 4;\n\t"
        "add.u32 x, %5, 4;\n\t"
        "or.b32 i, %3, 0;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], a, b, i, [s], [x], t;\n\t"
        "add.s64 a, %1, 6;\n\t"
        "add.s64 b, %2, 6;\n\t"
        "add.u32 s, %4, 4;\n\t"
        "add.u32 x, %5, 4;\n\t"
        "or.b32 i, %3, 1073741856;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], a, b, i, [s], [x], t;\n\t"
        "}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "l"(w_scales), "l"(x_scales), "r"(onto)
        : "memory");
  } else if constexpr (STRIPS == 2) {
    asm volatile(
        "{\n\t"
        ".reg .pred one, p, t;\n\t"
        ".reg .b32 s, x, i;\n\t"
        ".reg .b64 q, a, b;\n\t"
        "elect.sync _|one, 0xffffffff;\n\t"
        "setp.ne.u32 p, %8, 0;\n\t"
        "setp.eq.u32 t, 0, 0;\n\t"
        "add.u32 s, %4, 0;\n\t"
        "add.s64 q, %6, 0;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [s], q;\n\t"
        "add.u32 x, %5, 0;\n\t"
        "add.s64 q, %7, 0;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 x, %5, 4;\n\t"
        "add.s64 q, %7, 128;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 s, %4, 4;\n\t"
        "add.s64 q, %6, 32;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [s], q;\n\t"
        "add.u32 x, %5, 8;\n\t"
        "add.s64 q, %7, 32;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 x, %5, 12;\n\t"
        "add.s64 q, %7, 160;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 s, %4, 8;\n\t"
        "add.s64 q, %6, 64;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [s], q;\n\t"
        "add.u32 x, %5, 16;\n\t"
        "add.s64 q, %7, 64;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 x, %5, 20;\n\t"
        "add.s64 q, %7, 192;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 s, %4, 12;\n\t"
        "add.s64 q, %6, 96;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [s], q;\n\t"
        "add.u32 x, %5, 24;\n\t"
        "add.s64 q, %7, 96;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 x, %5, 28;\n\t"
        "add.s64 q, %7, 224;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.s64 a, %1, 0;\n\t"
        "add.s64 b, %2, 0;\n\t"
        "add.u32 s, %4, 0;\n\t"
        "add.u32 x, %5, 0;\n\t"
        "or.b32 i, %3, 0;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a, b, i, [s], [x], p;\n\t"
        "add.s64 a, %1, 2;\n\t"
        "add.s64 b, %2, 2;\n\t"
        "add.u32 s, %4, 4;\n\t"
        "add.u32 x, %5, 8;\n\t"
        "or.b32 i, %3, 0;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a, b, i, [s], [x], t;\n\t"
        "add.s64 a, %1, 4;\n\t"
        "add.s64 b, %2, 4;\n\t"
        "add.u32 s, %4, 8;\n\t"
        "add.u32 x, %5, 16;\n\t"
        "or.b32 i, %3, 0;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a, b, i, [s], [x], t;\n\t"
        "add.s64 a, %1, 6;\n\t"
        "add.s64 b, %2, 6;\n\t"
        "add.u32 s, %4, 12;\n\t"
        "add.u32 x, %5, 24;\n\t"
        "or.b32 i, %3, 0;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a, b, i, [s], [x], t;\n\t"
        "}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "l"(w_scales), "l"(x_scales), "r"(onto)
        : "memory");
  } else {
    asm volatile(
        "{\n\t"
        ".reg .pred one, p, t;\n\t"
        ".reg .b32 s, x, i;\n\t"
        ".reg .b64 q, a, b;\n\t"
        "elect.sync _|one, 0xffffffff;\n\t"
        "setp.ne.u32 p, %8, 0;\n\t"
        "setp.eq.u32 t, 0, 0;\n\t"
        "add.u32 s, %4, 0;\n\t"
        "add.s64 q, %6, 0;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [s], q;\n\t"
        "add.u32 x, %5, 0;\n\t"
        "add.s64 q, %7, 0;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 s, %4, 4;\n\t"
        "add.s64 q, %6, 32;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [s], q;\n\t"
        "add.u32 x, %5, 4;\n\t"
        "add.s64 q, %7, 32;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 s, %4, 8;\n\t"
        "add.s64 q, %6, 64;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [s], q;\n\t"
        "add.u32 x, %5, 8;\n\t"
        "add.s64 q, %7, 64;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.u32 s, %4, 12;\n\t"
        "add.s64 q, %6, 96;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [s], q;\n\t"
        "add.u32 x, %5, 12;\n\t"
        "add.s64 q, %7, 96;\n\t"
        "@one tcgen05.cp.cta_group::2.32x128b.warpx4 [x], q;\n\t"
        "add.s64 a, %1, 0;\n\t"
        "add.s64 b, %2, 0;\n\t"
        "add.u32 s, %4, 0;\n\t"
        "add.u32 x, %5, 0;\n\t"
        "or.b32 i, %3, 0;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a, b, i, [s], [x], p;\n\t"
        "add.s64 a, %1, 2;\n\t"
        "add.s64 b, %2, 2;\n\t"
        "add.u32 s, %4, 4;\n\t"
        "add.u32 x, %5, 4;\n\t"
        "or.b32 i, %3, 0;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a, b, i, [s], [x], t;\n\t"
        "add.s64 a, %1, 4;\n\t"
        "add.s64 b, %2, 4;\n\t"
        "add.u32 s, %4, 8;\n\t"
        "add.u32 x, %5, 8;\n\t"
        "or.b32 i, %3, 0;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a, b, i, [s], [x], t;\n\t"
        "add.s64 a, %1, 6;\n\t"
        "add.s64 b, %2, 6;\n\t"
        "add.u32 s, %4, 12;\n\t"
        "add.u32 x, %5, 12;\n\t"
        "or.b32 i, %3, 0;\n\t"
        "@one tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], a, b, i, [s], [x], t;\n\t"
        "}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "l"(w_scales), "l"(x_scales), "r"(onto)
        : "memory");
  }
}

// Whether tiles of 128 rows of x serve better than 256: they take three quarters of the time, so where there are not more rounds
// of them (256 tokens 4096 by 4096: 8.3 and 9.7 us, 64 tokens by 11008 8.1 and 9.3; 333 tokens 5119 by 13823, three rounds
// and two: 22.9 and 19.5).
inline bool narrow_tiles(int32_t x_rows, uint64_t w_tiles, int sm_count) {
  const uint64_t pairs = (uint64_t)sm_count / 2;
  const uint64_t rounds_256 = (w_tiles * (((uint64_t)x_rows + 255) / 256) + pairs - 1) / pairs;
  const uint64_t rounds_128 = (w_tiles * (((uint64_t)x_rows + 127) / 128) + pairs - 1) / pairs;
  return rounds_128 * 3 < rounds_256 * 4;
}

// Few tiles of many steps: two or four pairs to a tile, as long as all clusters run at once (those of eight blocks leave more
// SMs over).  By single pairs and so, 256 tokens 8192 by 4096 e4m3 13.5 and 11.3 us, 75 tokens 21892 by 2787 28.8 and 12.9; but
// 200 tokens 2048 by 2048 6.0 and 7.2, and four pairs to each of 16 tiles, 32 tokens 4096 by 4096, 7.7 and 11.3.
inline uint32_t pairs_per_tile(uint32_t tiles, uint32_t steps, int sm_count) {
  const uint32_t all = (uint32_t)sm_count / 2;
  if (tiles > all * 7 / 16 || steps < 2 * kLeastSteps) return 1;
  return tiles <= all / 6 && steps >= 4 * kLeastSteps ? 4 : 2;
}

}  // namespace
}  // namespace mx
}  // namespace pvt
#endif
