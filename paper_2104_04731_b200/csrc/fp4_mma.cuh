// Device code shared by the kernels that form products of 4-bit matrices on the tensor core (tcgen05.mma, block_scale).
//
// A stage is 256 elements of the reduction: 128 bytes of every row, four MMAs of depth 64.  The tensor core takes the scales from tensor
// memory: lane r, column c of a group of four columns holds four consecutive scales of row 32 c + r, for all four quarters of the lanes alike.
// In memory a row's scales follow each other, so a copy brings pieces of 128 rows; a warp turns them round in place (a lane has the pieces of four
// rows, 32 apart, and every group of columns takes a word of each) and tcgen05.cp carries 512 bytes to four columns.
#pragma once

#include "fp4_common.cuh"
#include "fp8_mma.cuh"

namespace b2c {

namespace {

constexpr int kStageRow = kFp4Stage / 2;  // bytes

// Instruction descriptor of kind::mxf4 and kind::mxf4nvf4: both operands E2M1 (code 1 at bits 7 and 10), N/8 at bit 17, kind of the scales (0 E4M3,
// 1 E8M0) at bit 23, M/16 at bit 24; the half of a scale word that an MMA uses at bits 29 and 4.
__device__ __forceinline__ uint32_t make_idesc_f4(int m, int n, int format) {
  return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((format == B2C_MXFP4 ? 1u : 0u) << 23) | ((uint32_t)(m >> 4) << 24);
}
constexpr uint32_t kUpperScales = (2u << 29) | (2u << 4);

// Descriptor of 32 lanes x 16 bytes in shared memory, rows of 8 x 16 bytes 128 apart.
__device__ __forceinline__ uint64_t make_scale_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFF) >> 4) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);
}
// A stage's scales of 128 rows to tensor memory: NV four, MX two times 512 bytes, `step` bytes apart, to four columns each, `columns` apart; with
// CTAS == 2 in both blocks of the pair, each from its own shared memory.  One asm block, so that the predicate is formed once and the
// instructions go out back to back: issuing them is what the tensor core waits for where the tiles are small.
template <int CTAS, int FORMAT, int STEP>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint32_t addr, int columns, uint32_t on) {
  const uint64_t desc = make_scale_desc(addr);
#define B2C_CP4(GROUP)                                                                                     \
  asm volatile(                                                                                            \
      "{\n.reg .pred q;\n.reg .b32 t1, t2, t3;\n.reg .b64 d1, d2, d3;\nsetp.ne.b32 q, %2, 0;\n"            \
      "add.u32 t1, %0, %3;\nadd.u32 t2, t1, %3;\nadd.u32 t3, t2, %3;\n"                                    \
      "add.u64 d1, %1, %4;\nadd.u64 d2, d1, %4;\nadd.u64 d3, d2, %4;\n"                                    \
      "@q tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [%0], %1;\n"                                      \
      "@q tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [t1], d1;\n"                                      \
      "@q tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [t2], d2;\n"                                      \
      "@q tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [t3], d3;\n}" ::"r"(taddr),                       \
      "l"(desc), "r"(on), "r"(columns), "n"(STEP >> 4)                                                     \
      : "memory")
#define B2C_CP2(GROUP)                                                                                     \
  asm volatile(                                                                                            \
      "{\n.reg .pred q;\n.reg .b32 t1;\n.reg .b64 d1;\nsetp.ne.b32 q, %2, 0;\n"                           \
      "add.u32 t1, %0, %3;\nadd.u64 d1, %1, %4;\n"                                                         \
      "@q tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [%0], %1;\n"                                      \
      "@q tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [t1], d1;\n}" ::"r"(taddr),                       \
      "l"(desc), "r"(on), "r"(columns), "n"(STEP >> 4)                                                     \
      : "memory")
  if constexpr (FORMAT == B2C_MXFP4) {
    if constexpr (CTAS == 1) B2C_CP2("1");
    else B2C_CP2("2");
  } else {
    if constexpr (CTAS == 1) B2C_CP4("1");
    else B2C_CP4("2");
  }
#undef B2C_CP4
#undef B2C_CP2
}
__host__ __device__ constexpr int stage_words(int format) { return format == B2C_MXFP4 ? 2 : 4; }  // groups of four columns, of a stage and 128 rows

// One stage: `ksteps` (1..4) MMAs over consecutive 32-byte slices; the first overwrites unless `accumulate`.  Scales of the A rows at
// sa, a group of four columns for one MMA (NV) or two (MX); of the B rows at sb, groups b_cols columns apart.
template <int CTAS, int FORMAT>
__device__ __forceinline__ void mma_f4_stage(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t b_cols,
                                             uint32_t accumulate, uint32_t on, int ksteps) {
#define B2C_F4_STAGE(GROUP, KIND, SA1, SA2, SA3, SB1, SB2, SB3, ID1)                                              \
  asm volatile(                                                                                                   \
      "{\n"                                                                                                       \
      ".reg .pred pacc, ptrue, q0, q1, q2, q3;\n"                                                                 \
      ".reg .b64 a1, a2, a3, b1, b2, b3;\n"                                                                       \
      "setp.ne.b32 pacc, %4, 0;\n"                                                                                \
      "setp.eq.b32 ptrue, 0, 0;\n"                                                                                \
      "setp.ne.b32 q0, %5, 0;\n"                                                                                  \
      "setp.gt.and.s32 q1, %6, 1, q0;\n"                                                                          \
      "setp.gt.and.s32 q2, %6, 2, q0;\n"                                                                          \
      "setp.gt.and.s32 q3, %6, 3, q0;\n"                                                                          \
      "add.u64 a1, %1, 2;\n"                                                                                      \
      "add.u64 b1, %2, 2;\n"                                                                                      \
      "add.u64 a2, %1, 4;\n"                                                                                      \
      "add.u64 b2, %2, 4;\n"                                                                                      \
      "add.u64 a3, %1, 6;\n"                                                                                      \
      "add.u64 b3, %2, 6;\n"                                                                                      \
      "@q0 tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %1, %2, %3, [%7], [%8], pacc;\n"                 \
      "@q1 tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], a1, b1, %9, [%10], [%11], ptrue;\n"              \
      "@q2 tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], a2, b2, %3, [%12], [%13], ptrue;\n"              \
      "@q3 tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], a3, b3, %9, [%14], [%15], ptrue;\n"              \
      "}" ::"r"(d_tmem),                                                                                          \
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(on), "r"(ksteps), "r"(sa), "r"(sb), "r"(ID1),      \
      "r"(SA1), "r"(SB1), "r"(SA2), "r"(SB2), "r"(SA3), "r"(SB3)                                                  \
      : "memory")
  if constexpr (FORMAT == B2C_MXFP4) {
    if constexpr (CTAS == 1) B2C_F4_STAGE("1", "mxf4.block_scale.scale_vec::2X", sa, sa + 4, sa + 4, sb, sb + b_cols, sb + b_cols, idesc | kUpperScales);
    else B2C_F4_STAGE("2", "mxf4.block_scale.scale_vec::2X", sa, sa + 4, sa + 4, sb, sb + b_cols, sb + b_cols, idesc | kUpperScales);
  } else {
    if constexpr (CTAS == 1) B2C_F4_STAGE("1", "mxf4nvf4.block_scale.scale_vec::4X", sa + 4, sa + 8, sa + 12, sb + b_cols, sb + 2 * b_cols, sb + 3 * b_cols, idesc);
    else B2C_F4_STAGE("2", "mxf4nvf4.block_scale.scale_vec::4X", sa + 4, sa + 8, sa + 12, sb + b_cols, sb + 2 * b_cols, sb + 3 * b_cols, idesc);
  }
#undef B2C_F4_STAGE
}

// Scales come for four stages at a time: 64 bytes (NV) or 32 (MX) of every row.  (The copy engine works by rows of a box: pieces of 16 bytes, a
// stage's, took it as long as the 128-byte rows of the operands.)
constexpr int kGroup = 4;
constexpr int kGroupTile = 128 * 64;  // bytes of a group's scales of 128 rows
inline __host__ __device__ int group_row(int format) { return format == B2C_MXFP4 ? 32 : 64; }

// A group's scales of up to 128 rows, as a copy with the swizzle of that width left them, turned round in place: word w of all rows
// becomes the 512 bytes at 512 w (NV: words 4 i .. 4 i + 3 are those of stage i, MX: 2 i and 2 i + 1).  A lane holds all of four rows, 32
// apart.  Called by a whole warp; what follows in the asynchronous proxy sees it after the caller's barrier.
template <int WORDS>
__device__ __forceinline__ void turn_group_words(uint32_t base, int rows, int lane) {
  uint32_t w[4][WORDS];
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int r = 32 * g + lane, x = WORDS == 16 ? (r >> 1) & 3 : (r >> 2) & 1;
#pragma unroll
    for (int c = 0; c < WORDS / 4; ++c) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[g][4 * c + j] = 0;
      if (32 * g < rows)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[g][4 * c]), "=r"(w[g][4 * c + 1]), "=r"(w[g][4 * c + 2]), "=r"(w[g][4 * c + 3])
                     : "r"(base + (uint32_t)(r * (4 * WORDS) + ((c ^ x) << 4)))
                     : "memory");
    }
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < WORDS; ++i)
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + (uint32_t)(512 * i + lane * 16)), "r"(w[0][i]), "r"(w[1][i]), "r"(w[2][i]), "r"(w[3][i]) : "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
__device__ __forceinline__ void turn_group(uint32_t base, int rows, int format, int lane) {
  if (format == B2C_MXFP4) turn_group_words<8>(base, rows, lane);
  else turn_group_words<16>(base, rows, lane);
}

__device__ __forceinline__ float alpha_of(const Matmul4Args& a, int group) {
  return (a.alpha != nullptr ? a.alpha[group] : 1.0f) * (a.alpha2 != nullptr ? *a.alpha2 : 1.0f);
}

}  // namespace
}  // namespace b2c
