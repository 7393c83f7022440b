// The cache held in 4 bits: layout of a tile of 64 rows of one (sequence, kv head), shared by the kernels that fill and read it.
//
// A tile is one run of bytes: key codes, value codes, key scales, value scales.  Inside it the codes lie in the lanes that the matrix
// instructions take their values from, so that a wave loads its operands with 16 bytes per lane, 1 KB in a piece, and moves nothing
// between lanes:
//   key codes    [16 rows][block of 32 elements][row] 16 bytes: word i of a lane's is its eight elements of the i-th 16x16x32 multiply
//   value codes  [chunk][lane][4] words: word w = 4 chunk + place is elements 16 (w / 2) .. + 15 of rows 32 (w % 2) .. + 31; the
//                lane's element is lane % 16, and its eight codes are rows 4 (lane / 16) + {0 .. 3} and the same + 16: the
//                order in which the lane holds the weights of those rows after the key multiply
//   key scales   [block][row % 16][row / 16] bytes: a lane's word holds the scales of its four key operands
//   value scales [row % 16 / 4][row / 16][row % 4] bytes: a lane's 16 bytes are those of the rows whose weights it holds
// Scales are the exponent + 127; 255 marks a row that is not a number.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fc_internal.h"

#define FC_Q4_K_LOWEST (-100)  // least exponent of a key block: nothing of the format is subnormal in fp32 or bfloat16
#define FC_Q4_V_LOWEST (-40)   // and of a value row: with the bound below, weights of rows 80 powers of two apart stay in range
#define FC_Q4_V_MOST 0x54c00000u  // 6 * 2^40 as a float
#define FC_Q4_K_MOST 0x7cc00000u  // 6 * 2^120: twice that could round to what no float holds

__host__ __device__ constexpr int fc_q4_tile_bytes(int dh) { return 64 * dh + 2 * dh + 64; }
__host__ __device__ constexpr int fc_q4_v(int dh) { return 32 * dh; }
__host__ __device__ constexpr int fc_q4_vscale(int dh) { return 66 * dh; }
__host__ __device__ constexpr int fc_q4_k_block(int dh, int r, int c) { return r / 16 * (8 * dh) + (c * 16 + r % 16) * 16; }
__host__ __device__ constexpr int fc_q4_kscale(int dh, int r, int c) { return 64 * dh + (c * 16 + r % 16) * 4 + r / 16; }
__host__ __device__ constexpr int fc_q4_vscale_at(int r) { return r % 16 / 4 * 16 + r / 16 * 4 + r % 4; }

// The value of a code, and of a scale byte.
__device__ __forceinline__ float fc_q4_value(uint32_t code)
{
    const uint32_t m = code & 7;
    const float a = m < 4 ? 0.5f * m : m < 6 ? (float)(m - 2) : (float)(2 * m - 8);
    return code & 8 ? -a : a;
}
__device__ __forceinline__ float fc_q4_scale(uint32_t byte) { return byte == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float(byte << 23); }

struct FcQ4Geom {
    int32_t B, Hq, Hkv, Dh, max_seq, spad, g, dtype;
    float scale;  // softmax scale
};

hipError_t fc_launch_q4_store(const FcQ4Geom &G, uint8_t *layer, const void *k, const void *v, const int32_t *pos, int start, int rows,
                              int src_spad, hipStream_t s);
hipError_t fc_launch_q4_read(const FcQ4Geom &G, const uint8_t *layer, void *k, void *v, int start, int rows, hipStream_t s);

// Launch plan of the attention (host, pure function of the shape).
struct FcQ4Plan {
    int rt;      // 16-row tiles of query rows a workgroup holds
    int waves;   // its waves
    int splits;  // ranges the keys are cut into
};
FcQ4Plan fc_plan_q4(const FcQ4Geom &G, int A, int kv_len, size_t cap);  // cap: bytes of partial results
size_t fc_q4_plan_workspace(const FcQ4Geom &G, const FcQ4Plan &p, int A);
size_t fc_q4_most_workspace(const FcQ4Geom &G, int max_rows);
hipError_t fc_launch_q4_attention(const FcQ4Geom &G, const FcQ4Plan &pl, const void *q, const uint8_t *layer, const int32_t *pos, const int32_t *lens, int A, int kv_len,
                                  void *out, void *workspace, hipStream_t s);
