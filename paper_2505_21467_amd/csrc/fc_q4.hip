// Rows of keys and values held in 4 bits: the tiles they are kept in, storing rows and reading them back.
//
// A value is an E2M1 number (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives) times a power of two: a key row has one power per
// block of 32 elements, which is what the matrix instructions with block scales take, a value row one for all its elements, which
// the attention multiplies the row's weight by instead of the row.  The power is the least one with which the block's largest
// magnitude is at most 6, so nothing is clipped, and x 2^-e is exact: the only rounding is the one to E2M1 (nearest, ties to the
// even code), which makes what is stored the same bits whoever computes it.
#include "fc_device.h"
#include "fc_internal.h"
#include "fc_q4.h"

namespace {

struct Q4Place {
    const int32_t *pos;  // nullptr: start + r
    int start, rows;
};

// Source of the rows: plain arrays [B][Hkv][rows][DH], or a layer of a full-precision cache, row by place.
template <typename T, int DH, bool FROM_CACHE>
__device__ __forceinline__ void q4_load32(const T *base, size_t pair, int rows_or_spad, int row, int d0, bool value, float (&x)[32])
{
    if (FROM_CACHE && value) {  // 64-row tiles, key index fastest
        const T *p = base + pair * (size_t)rows_or_spad * DH + (size_t)(row / FC_VTILE) * (FC_VTILE * DH) + (size_t)d0 * FC_VTILE + row % FC_VTILE;
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = fc_to_float(p[(size_t)i * FC_VTILE]);
        return;
    }
    const T *p = base + (pair * (size_t)rows_or_spad + row) * DH + d0;
    constexpr int PER = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 32 / PER; ++i) {
        struct piece { T v[PER]; };
        const piece v = __builtin_bit_cast(piece, fc_load_any<uint4>(p + i * PER));
#pragma unroll
        for (int j = 0; j < PER; ++j) x[i * PER + j] = fc_to_float(v.v[j]);
    }
}

// Largest magnitude as raw bits: NaN and infinity come out above every finite number.
__device__ __forceinline__ uint32_t q4_top(const float (&x)[32])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    return m;
}

// The least e >= lowest with top <= 6 2^e.  6 = 1.5 * 2^2: the exponent of top less two, or one more where its fraction is above a half.
__device__ __forceinline__ int q4_exponent(uint32_t top, int lowest)
{
    const int e = (int)(top >> 23) - 127 - 2 + ((top & 0x7fffffu) > 0x400000u ? 1 : 0);
    return max(e, lowest);
}

// 32 values by 2^-e to E2M1, eight codes a word, the lower four bits first.
__device__ __forceinline__ void q4_codes(const float (&x)[32], int e, uint32_t (&w)[4])
{
    const float s = __uint_as_float((uint32_t)(e + 127) << 23);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[8 * i], x[8 * i + 1], s, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[8 * i + 2], x[8 * i + 3], s, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[8 * i + 4], x[8 * i + 5], s, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[8 * i + 6], x[8 * i + 7], s, 3);
        w[i] = c;
    }
}

// One workgroup owns one tile of 64 places of one (sequence, kv head): a word of value codes holds eight places, so no two
// workgroups may write one.  With a list of places the workgroup of an entry steps back if an earlier entry names the same tile.
// Where a place is listed twice, the later entry is the one stored.
//
// Bound by memory where there is much to store (16384 rows of 4 heads, 33.6 MB in and 8.7 MB out); a block is one latency chain.
template <typename T, int DH, bool FROM_CACHE>
__global__ __launch_bounds__(2 * DH) void k_q4_store(uint8_t *layer, const T *__restrict__ k, const T *__restrict__ v, Q4Place p, int max_seq,
                                                  int tiles, int rows_or_spad, int Hkv)
{
    constexpr int C = DH / 32;                // blocks of a row, a thread each
    constexpr int THREADS = FC_VTILE * C;     // (= 2 DH)
    constexpr int PITCH = DH + 4;             // bytes of a row of value codes, one code a byte
    __shared__ int s_src[FC_VTILE];
    __shared__ __align__(16) uint8_t s_code[FC_VTILE * PITCH];
    const int tid = threadIdx.x;
    const size_t pair = blockIdx.y;
    const int b = (int)(pair / Hkv);
    int tile;
    if (tid < FC_VTILE) s_src[tid] = -1;
    if (p.pos) {
        const int32_t *pos = p.pos + (size_t)b * p.rows;
        const int mine = pos[blockIdx.x];
        if (mine < 0 || mine >= max_seq) return;  // (the whole workgroup)
        tile = mine / FC_VTILE;
        int found = 0;
        for (int a = tid; a < (int)blockIdx.x; a += THREADS) {
            const int o = pos[a];
            found |= o >= 0 && o < max_seq && o / FC_VTILE == tile;
        }
        if (__syncthreads_or(found)) return;
        for (int a = (int)blockIdx.x + tid; a < p.rows; a += THREADS) {
            const int o = pos[a];
            if (o >= 0 && o < max_seq && o / FC_VTILE == tile) atomicMax(&s_src[o % FC_VTILE], a);
        }
    } else {
        tile = p.start / FC_VTILE + blockIdx.x;
        __syncthreads();
        if (tid < FC_VTILE) {
            const int r = tile * FC_VTILE + tid - p.start;
            if (r >= 0 && r < p.rows) s_src[tid] = r;
        }
    }
    __syncthreads();
    uint8_t *rec = layer + (pair * tiles + tile) * (size_t)fc_q4_tile_bytes(DH);
    uint8_t *vs = rec + fc_q4_vscale(DH);
    const int r = tid / C, c = tid % C, src = s_src[r];
    if (src >= 0) {
        const int from = FROM_CACHE ? tile * FC_VTILE + r : src;
        float x[32];
        uint32_t w[4];
        q4_load32<T, DH, FROM_CACHE>(v, pair, rows_or_spad, from, 32 * c, true, x);
        uint32_t top_v = q4_top(x);
        float y[32];
        q4_load32<T, DH, FROM_CACHE>(k, pair, rows_or_spad, from, 32 * c, false, y);
        const uint32_t top_k = q4_top(y);
        uint32_t all_k = top_k;
#pragma unroll
        for (int o = 1; o < C; o <<= 1) {  // (the blocks of a row are neighbouring lanes, all of them here)
            top_v = max(top_v, (uint32_t)__shfl_xor((int)top_v, o));
            all_k = max(all_k, (uint32_t)__shfl_xor((int)all_k, o));
        }
        const bool bad = all_k > FC_Q4_K_MOST || top_v > FC_Q4_V_MOST;
        const int ev = q4_exponent(top_v, FC_Q4_V_LOWEST), ek = q4_exponent(top_k, FC_Q4_K_LOWEST);
        q4_codes(x, bad ? 0 : ev, w);
        uint32_t *code = (uint32_t *)(s_code + r * PITCH + 32 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = bad ? 0 : w[i];
            code[2 * i] = (u & 0xf) | (u & 0xf0) << 4 | (u & 0xf00) << 8 | (u & 0xf000) << 12;
            code[2 * i + 1] = (u >> 16 & 0xf) | (u >> 16 & 0xf0) << 4 | (u >> 16 & 0xf00) << 8 | (u >> 16 & 0xf000) << 12;
        }
        q4_codes(y, bad ? 0 : ek, w);
        if (bad) w[0] = w[1] = w[2] = w[3] = 0;
        *(uint4 *)(rec + fc_q4_k_block(DH, r, c)) = make_uint4(w[0], w[1], w[2], w[3]);
        rec[fc_q4_kscale(DH, r, c)] = bad ? 255 : (uint8_t)(ek + 127);
        if (c == 0) vs[fc_q4_vscale_at(r)] = bad ? 255 : (uint8_t)(ev + 127);
    }
    __syncthreads();
    // Value codes: a word is eight places of one element, in the order in which the attention's multiplies take them.
    uint32_t *words = (uint32_t *)(rec + fc_q4_v(DH));
#pragma unroll 1
    for (int i = tid; i < 8 * DH; i += THREADS) {  // i: chunk, lane, word of the chunk
        const int lane = i / 4 % 64, w = i / 256 * 4 + i % 4, d = w / 2 * 16 + lane % 16, r0 = w % 2 * 32 + lane / 16 * 4;
        uint32_t code = 0, keep = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = r0 + j / 4 * 16 + j % 4;
            if (s_src[row] >= 0) code |= (uint32_t)s_code[row * PITCH + d] << (4 * j);
            else keep |= 0xfu << (4 * j);
        }
        if (keep == 0xffffffffu) continue;
        if (keep) code |= words[i] & keep;
        words[i] = code;
    }
}

// Rows [start, start + rows) back as the values they stand for; one workgroup per tile.
template <typename T, int DH>
__global__ __launch_bounds__(2 * DH) void k_q4_read(const uint8_t *layer, T *__restrict__ k, T *__restrict__ v, int start, int rows, int tiles)
{
    constexpr int C = DH / 32, PITCH = DH + 4, THREADS = FC_VTILE * C;
    __shared__ __align__(16) uint8_t s_code[FC_VTILE * PITCH];
    const int tid = threadIdx.x, tile = start / FC_VTILE + blockIdx.x;
    const size_t pair = blockIdx.y;
    const uint8_t *rec = layer + (pair * tiles + tile) * (size_t)fc_q4_tile_bytes(DH);
    const uint32_t *words = (const uint32_t *)(rec + fc_q4_v(DH));
    for (int i = tid; i < 8 * DH; i += THREADS) {
        const int lane = i / 4 % 64, w = i / 256 * 4 + i % 4, d = w / 2 * 16 + lane % 16, r0 = w % 2 * 32 + lane / 16 * 4;
        const uint32_t code = words[i];
#pragma unroll
        for (int j = 0; j < 8; ++j) s_code[(r0 + j / 4 * 16 + j % 4) * PITCH + d] = code >> (4 * j) & 0xf;
    }
    __syncthreads();
    const int r = tid / C, c = tid % C, to = tile * FC_VTILE + r - start;
    if (to >= 0 && to < rows) {
        const size_t at = (pair * (size_t)rows + to) * DH + 32 * c;
        const uint4 kc = *(const uint4 *)(rec + fc_q4_k_block(DH, r, c));
        const uint32_t kw[4] = {kc.x, kc.y, kc.z, kc.w};
        const float ks = fc_q4_scale(rec[fc_q4_kscale(DH, r, c)]), vsc = fc_q4_scale(rec[fc_q4_vscale(DH) + fc_q4_vscale_at(r)]);
        const uint32_t *vc = (const uint32_t *)(s_code + r * PITCH + 32 * c);
        constexpr int PER = 16 / sizeof(T);
        struct piece { T x[PER]; };
#pragma unroll
        for (int i = 0; i < 32; i += PER) {
            piece a, o;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                a.x[j] = fc_from_float<T>(fc_q4_value(kw[(i + j) / 8] >> (4 * ((i + j) % 8)) & 0xf) * ks);
                o.x[j] = fc_from_float<T>(fc_q4_value(vc[(i + j) / 4] >> (8 * ((i + j) % 4)) & 0xf) * vsc);
            }
            fc_store_any(k + at + i, __builtin_bit_cast(uint4, a));
            fc_store_any(v + at + i, __builtin_bit_cast(uint4, o));
        }
    }
}

template <typename T, int DH>
void launch_store(const FcQ4Geom &G, uint8_t *layer, const void *k, const void *v, const int32_t *pos, int start, int rows, int src_spad,
                  hipStream_t s)
{
    const int tiles = G.spad / FC_VTILE;
    const int n = pos ? rows : (start + rows - 1) / FC_VTILE - start / FC_VTILE + 1;
    const dim3 grid((unsigned)n, (unsigned)(G.B * G.Hkv));
    const Q4Place p{pos, start, rows};
    if (src_spad)
        k_q4_store<T, DH, true><<<grid, dim3(2 * DH), 0, s>>>(layer, (const T *)k, (const T *)v, p, G.max_seq, tiles, src_spad, G.Hkv);
    else
        k_q4_store<T, DH, false><<<grid, dim3(2 * DH), 0, s>>>(layer, (const T *)k, (const T *)v, p, G.max_seq, tiles, rows, G.Hkv);
}

template <typename T, int DH>
void launch_read(const FcQ4Geom &G, const uint8_t *layer, void *k, void *v, int start, int rows, hipStream_t s)
{
    const dim3 grid((unsigned)((start + rows - 1) / FC_VTILE - start / FC_VTILE + 1), (unsigned)(G.B * G.Hkv));
    k_q4_read<T, DH><<<grid, dim3(2 * DH), 0, s>>>(layer, (T *)k, (T *)v, start, rows, G.spad / FC_VTILE);
}

}  // namespace

// src_spad: rows a (sequence, kv head) has in the full-precision cache that is the source; 0: plain arrays.
hipError_t fc_launch_q4_store(const FcQ4Geom &G, uint8_t *layer, const void *k, const void *v, const int32_t *pos, int start, int rows,
                              int src_spad, hipStream_t s)
{
    if (G.dtype == FC_F32) {
        if (G.Dh == 128) launch_store<float, 128>(G, layer, k, v, pos, start, rows, src_spad, s);
        else launch_store<float, 64>(G, layer, k, v, pos, start, rows, src_spad, s);
    } else {
        if (G.Dh == 128) launch_store<bf16_t, 128>(G, layer, k, v, pos, start, rows, src_spad, s);
        else launch_store<bf16_t, 64>(G, layer, k, v, pos, start, rows, src_spad, s);
    }
    return hipGetLastError();
}

hipError_t fc_launch_q4_read(const FcQ4Geom &G, const uint8_t *layer, void *k, void *v, int start, int rows, hipStream_t s)
{
    if (G.dtype == FC_F32) {
        if (G.Dh == 128) launch_read<float, 128>(G, layer, k, v, start, rows, s);
        else launch_read<float, 64>(G, layer, k, v, start, rows, s);
    } else {
        if (G.Dh == 128) launch_read<bf16_t, 128>(G, layer, k, v, start, rows, s);
        else launch_read<bf16_t, 64>(G, layer, k, v, start, rows, s);
    }
    return hipGetLastError();
}
