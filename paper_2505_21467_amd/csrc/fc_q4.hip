// Rows of keys and values held in 4 bits: the tiles they are kept in, storing rows and reading them back.
//
// A value is an E2M1 number (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives) times a power of two: a key row has one power per
// block of 32 elements (channels of very different sizes stay apart), a value row one for all its elements, which
// the attention multiplies the row's weight by instead of the row.  The power is the least one with which the block's largest
// magnitude is at most 6, so nothing is clipped, and x 2^-e is exact: the only rounding is the one to E2M1 (nearest, ties to the
// even code), which makes what is stored the same bits whoever computes it.
#include "fc_device.h"
#include "fc_internal.h"
#include "fc_q4.h"

namespace {

struct Q4Place {
    const int32_t *pos;  // nullptr: start + r
    int start, rows, by_entry;
};

// Eight neighbouring elements, and as floats.
template <typename T>
struct Eight {
    uint4 raw[sizeof(T) / 2];
    template <bool ONCE>  // with the non-temporal hint
    __device__ __forceinline__ void load(const T *p)
    {
        typedef uint32_t any __attribute__((ext_vector_type(4), aligned(2)));
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const T *at = p + i * 16 / sizeof(T);
            raw[i] = ONCE ? __builtin_bit_cast(uint4, __builtin_nontemporal_load((const any *)at)) : fc_load_any<uint4>(at);
        }
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        struct list { T v[8]; };
        const list l = __builtin_bit_cast(list, *this);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fc_to_float(l.v[i]);
    }
};

// Largest magnitude as raw bits: NaN and infinity come out above every finite number.
__device__ __forceinline__ uint32_t q4_top(const float (&x)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    return m;
}

// The least e >= lowest with top <= 6 2^e.  6 = 1.5 * 2^2: the exponent of top less two, or one more where its fraction is above a half.
__device__ __forceinline__ int q4_exponent(uint32_t top, int lowest)
{
    const int e = (int)(top >> 23) - 127 - 2 + ((top & 0x7fffffu) > 0x400000u ? 1 : 0);
    return max(e, lowest);
}

// Eight values by 2^-e to E2M1, the lower four bits first.
__device__ __forceinline__ uint32_t q4_codes(const float (&x)[8], int e)
{
    const float s = __uint_as_float((uint32_t)(e + 127) << 23);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
}

// Eight words of eight codes, the other way round: code j of word i for code i of word j.
__device__ __forceinline__ void q4_transpose(uint32_t (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = x[i], b = x[i + 4];
        x[i] = __builtin_amdgcn_perm(b, a, 0x05040100);
        x[i + 4] = __builtin_amdgcn_perm(b, a, 0x07060302);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int i = k / 2 * 4 + k % 2;
        const uint32_t a = x[i], b = x[i + 2];
        x[i] = __builtin_amdgcn_perm(b, a, 0x06020400);
        x[i + 2] = __builtin_amdgcn_perm(b, a, 0x07030501);
    }
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const uint32_t a = x[i], b = x[i + 1];
        x[i] = (a & 0x0f0f0f0fu) | (b & 0x0f0f0f0fu) << 4;
        x[i + 1] = (a >> 4 & 0x0f0f0f0fu) | (b & 0xf0f0f0f0u);
    }
}

// A tile in LDS.  A workgroup has 2 DH threads: one for every 16 bytes of key codes and of value codes, or 16 rows at a time with eight elements
// a thread.  Value codes turn between words of a row (eight elements) and words of the tile (eight rows) in DH threads, 8 x 8 codes each.
template <int DH>
struct Q4Tile {
    static constexpr int LANES = DH / 8, PITCH = LANES + 4, SCALES = 2 * DH + 64;
    uint4 k[2 * DH], v[2 * DH];
    uint32_t row[FC_VTILE * PITCH];  // value codes of a row
    __align__(16) uint8_t scale[SCALES];

    // (pieces of value codes are moved within their eight so that the turning threads meet in no bank)
    static __device__ __forceinline__ int place(int piece) { return piece ^ (piece >> 3 & 7); }
    __device__ __forceinline__ uint32_t &value_word(int piece, int i) { return ((uint32_t *)v)[place(piece) * 4 + i]; }
    __device__ __forceinline__ uint32_t &key_word(int r, int i) { return ((uint32_t *)k)[fc_q4_k_block(DH, r, i / 4) / 4 + i % 4]; }
    __device__ __forceinline__ uint8_t &key_scale(int r, int c) { return scale[fc_q4_kscale(DH, r, c) - 64 * DH]; }
    __device__ __forceinline__ uint8_t &value_scale(int r) { return scale[2 * DH + fc_q4_vscale_at(r)]; }

    // Thread t < DH: bits of t are half of the rows, word of the piece, half of the sixteen elements, four rows of sixteen (2), piece.
    template <bool STORE>
    __device__ __forceinline__ void turn(int t)
    {
        const int half = t & 1, g = t >> 3 & 3, chunk = t >> 5, word = chunk * 4 + (t >> 1 & 1) * 2 + (t >> 2 & 1);
        const int piece = chunk * 64 + g * 16 + (t >> 2 & 1) * 8, r0 = half * 32 + g * 4;
        uint32_t x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = STORE ? row[(r0 + i / 4 * 16 + i % 4) * PITCH + word] : value_word(piece + i, t & 3);
        q4_transpose(x);
#pragma unroll
        for (int i = 0; i < 8; ++i) (STORE ? value_word(piece + i, t & 3) : row[(r0 + i / 4 * 16 + i % 4) * PITCH + word]) = x[i];
    }
};

// One bit to four.
__device__ __forceinline__ uint32_t q4_spread(uint32_t x)
{
    x = (x | x << 12) & 0x000f000fu;
    x = (x | x << 6) & 0x03030303u;
    x = (x | x << 3) & 0x11111111u;
    return x * 15;
}

// One workgroup owns one tile of 64 places of one (sequence, kv head): a word of value codes holds eight places, so no two
// workgroups may write one.  With a list of places there is a workgroup for every entry, which steps back if an earlier entry names the same tile, or,
// where that is fewer, for every tile.  Where a place is listed twice, the later entry is the one stored.
//
// The source is plain arrays [B][Hkv][rows][DH] or a layer of a full-precision cache, row by place: keys alike, values [DH][64] by tiles, of which a
// thread takes the eight rows of a word of the tile, so that nothing is turned.
//
// Bound by memory where there is much to store; a block is one latency chain.  All that a thread loads is in flight at once, 16 bytes a lane next to
// one another on both sides.  4 x 32 heads x 4096 rows from HBM (268 MB in, 71 MB out) take 54 us with the non-temporal hint (ONCE: rows that exceed the
// memory-side cache) and 80 .. 88 without; reading them back 56 .. 64, 5.4 TB/s and more, where a large copy reaches 4.9.  4 x 8192 rows in
// fp32 that are in that cache: 8.7 us without the hint, 10.1 with it.  A block of 32 elements a thread and a byte per value code in LDS took
// 107 us each way.  19 entries: 5 us.
template <typename T, int DH, bool FROM_CACHE, bool ONCE>
__global__ __launch_bounds__(2 * DH) void k_q4_store(uint8_t *layer, const T *__restrict__ k, const T *__restrict__ v, Q4Place p, int max_seq,
                                                  int tiles, int rows_or_spad, int Hkv)
{
    using Tile = Q4Tile<DH>;
    constexpr int THREADS = 2 * DH, LANES = Tile::LANES, PASSES = FC_VTILE * LANES / THREADS, STEP = FC_VTILE / PASSES;
    __shared__ Tile s;
    __shared__ int s_src[FC_VTILE];
    __shared__ uint32_t s_top[FC_VTILE], s_bad[FC_VTILE];
    const int tid = threadIdx.x;
    const size_t pair = blockIdx.y;
    int tile;
    uint64_t stored;
    if (FROM_CACHE && tid < FC_VTILE) s_top[tid] = 0;
    if (p.pos) {
        const int32_t *pos = p.pos + (pair / Hkv) * p.rows;
        if (tid < FC_VTILE) s_src[tid] = -1;
        int first = 0;
        if (p.by_entry) {
            first = (int)blockIdx.x;
            const int mine = pos[first];
            if (mine < 0 || mine >= max_seq) return;  // (the whole workgroup)
            tile = mine / FC_VTILE;
            int found = 0;
            for (int a = tid; a < first; a += THREADS) {
                const int o = pos[a];
                found |= o >= 0 && o < max_seq && o / FC_VTILE == tile;
            }
            if (__syncthreads_or(found)) return;
        } else {
            tile = (int)blockIdx.x;
            __syncthreads();
        }
        for (int a = first + tid; a < p.rows; a += THREADS) {
            const int o = pos[a];
            if (o >= 0 && o < max_seq && o / FC_VTILE == tile) atomicMax(&s_src[o % FC_VTILE], a);
        }
        __syncthreads();
        stored = __ballot(s_src[tid % 64] >= 0);
        if (!stored) return;
    } else {
        tile = p.start / FC_VTILE + blockIdx.x;
        const int from = max(p.start - tile * FC_VTILE, 0), to = min(p.start + p.rows - tile * FC_VTILE, FC_VTILE);
        stored = (~0ull >> (64 - to)) & (~0ull << from);
        if (FROM_CACHE) __syncthreads();
    }
    uint8_t *rec = layer + (pair * tiles + tile) * (size_t)fc_q4_tile_bytes(DH);
    uint4 *rec_v = (uint4 *)(rec + fc_q4_v(DH)) + tid;
    uint32_t *rec_scale = (uint32_t *)(rec + 64 * DH) + tid;
    const bool whole = stored == ~0ull, scales = tid < Tile::SCALES / 4;

    const int lane = tid % LANES, r0 = tid / LANES;
    Eight<T> kx[PASSES], vx[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int r = r0 + i * STEP;
        // (rows that are not stored: another one's elements)
        const int src = FROM_CACHE ? tile * FC_VTILE + r : p.pos ? max(s_src[r], 0) : min(max(tile * FC_VTILE + r - p.start, 0), p.rows - 1);
        const size_t at = (pair * (size_t)rows_or_spad + src) * DH + lane * 8;
        kx[i].template load<ONCE>(k + at);
        if (!FROM_CACHE) vx[i].template load<ONCE>(v + at);
    }
    struct __align__(4 * sizeof(T)) Four { T v[4]; };  // (the cache's values: aligned)
    Four four[PASSES][2];
    const int half = tid & 1, g = tid >> 1 & 3, vr = half * 32 + g * 4, d0 = tid / 8;  // FROM_CACHE: rows vr + {0 .. 3, 16 .. 19} of elements d0 + 2 DH / 8 i
    if (FROM_CACHE) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                four[i][j] = *(const Four *)(v + pair * (size_t)rows_or_spad * DH + (size_t)tile * (FC_VTILE * DH) + (d0 + THREADS / 8 * i) * FC_VTILE + vr + 16 * j);
    }
    uint4 old = make_uint4(0, 0, 0, 0);
    uint32_t old_scale = 0;
    if (!whole) {
        old = *rec_v;
        if (scales) old_scale = *rec_scale;
    }

    uint32_t kw[PASSES];
    int ek[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int r = r0 + i * STEP;
        float x[8];
        kx[i].get(x);
        uint32_t top = q4_top(x);  // (the four lanes of a block are neighbours, and so are the lanes of a row)
        top = max(top, (uint32_t)__shfl_xor((int)top, 1));
        top = max(top, (uint32_t)__shfl_xor((int)top, 2));
        ek[i] = q4_exponent(top, FC_Q4_K_LOWEST);
        kw[i] = q4_codes(x, ek[i]);
#pragma unroll
        for (int o = 4; o < LANES; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        bool bad = top > FC_Q4_K_MOST;
        if (FROM_CACHE) {
            if (lane == 0) s_bad[r] = bad;
            continue;
        }
        vx[i].get(x);
        top = q4_top(x);
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        bad |= top > FC_Q4_V_MOST;
        const int ev = q4_exponent(top, FC_Q4_V_LOWEST);
        const uint32_t w = q4_codes(x, ev);
        s.row[r * Tile::PITCH + lane] = bad ? 0 : w;
        s.key_word(r, lane) = bad ? 0 : kw[i];
        if (lane % 4 == 0) s.key_scale(r, lane / 4) = bad ? 255 : (uint8_t)(ek[i] + 127);
        if (lane == 0) s.value_scale(r) = bad ? 255 : (uint8_t)(ev + 127);
    }
    if (FROM_CACHE) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) top = max(top, __float_as_uint(fc_to_float(four[i][j / 4].v[j % 4])) & 0x7fffffffu);
#pragma unroll
            for (int o = 8; o < 64; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
            if (tid % 64 < 8) atomicMax(&s_top[vr + j / 4 * 16 + j % 4], top);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int r = r0 + i * STEP;
            const bool bad = s_bad[r] || s_top[r] > FC_Q4_V_MOST;
            s.key_word(r, lane) = bad ? 0 : kw[i];
            if (lane % 4 == 0) s.key_scale(r, lane / 4) = bad ? 255 : (uint8_t)(ek[i] + 127);
            if (lane == 0) s.value_scale(r) = bad ? 255 : (uint8_t)(q4_exponent(s_top[r], FC_Q4_V_LOWEST) + 127);
        }
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = vr + j / 4 * 16 + j % 4;
            const uint32_t top = s_top[r];
            // (0: a row that is not a number, or too large)
            f[j] = s_bad[r] || top > FC_Q4_V_MOST ? 0.f : __uint_as_float((uint32_t)(127 - q4_exponent(top, FC_Q4_V_LOWEST)) << 23);
        }
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int d = d0 + THREADS / 8 * i, w = d / 16 * 2 + half;
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = f[j] == 0.f ? 0.f : fc_to_float(four[i][j / 4].v[j % 4]) * f[j];
            s.value_word(w / 4 * 64 + g * 16 + d % 16, w % 4) = q4_codes(x, 0);
        }
    } else {
        __syncthreads();
        if (tid < DH) s.template turn<true>(tid);
    }
    __syncthreads();
    uint4 now = s.v[Tile::place(tid)];
    if (!whole) {  // the rows of a word: four bits of `stored` at g, and four 16 further on; the second and fourth word's 32 further
        const uint64_t m = stored >> (tid / 16 % 4 * 4);
        const uint32_t a = q4_spread((uint32_t)(m & 15) | (uint32_t)(m >> 16 & 15) << 4), b = q4_spread((uint32_t)(m >> 32 & 15) | (uint32_t)(m >> 48 & 15) << 4);
        now = make_uint4((now.x & a) | (old.x & ~a), (now.y & b) | (old.y & ~b), (now.z & a) | (old.z & ~a), (now.w & b) | (old.w & ~b));
    }
    *rec_v = now;
    if (stored >> (tid / (DH / 2) * 16 + tid % 16) & 1) ((uint4 *)rec)[tid] = s.k[tid];
    if (scales) {
        uint32_t m = 0;  // the bytes of this word whose rows are stored
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int w = tid - DH / 2, r = w < 0 ? i * 16 + tid % 16 : w % 4 * 16 + w / 4 * 4 + i;
            if (stored >> r & 1) m |= 0xffu << (8 * i);
        }
        *rec_scale = (((const uint32_t *)s.scale)[tid] & m) | (old_scale & ~m);
    }
}

// Eight codes times 2^(byte - 127), in T (exact in either type).
__device__ __forceinline__ void q4_put(bf16_t *to, uint32_t c, uint32_t byte)
{
    uint4 x;
    if (byte == 255) {
        x = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
    } else {
        const float s = fc_q4_scale(byte);
        x.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((int)c, s, 0));
        x.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((int)c, s, 1));
        x.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((int)c, s, 2));
        x.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((int)c, s, 3));
    }
    fc_store_any(to, x);
}
__device__ __forceinline__ void q4_put(float *to, uint32_t c, uint32_t byte)
{
    const float s = fc_q4_scale(byte);  // (not a number for 255)
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fc_q4_value(c >> (4 * i)) * s;
    fc_store_any(to, make_float4(x[0], x[1], x[2], x[3]));
    fc_store_any(to + 4, make_float4(x[4], x[5], x[6], x[7]));
}

// Rows [start, start + rows) back as the values they stand for; one workgroup per tile.
template <typename T, int DH>
__global__ __launch_bounds__(2 * DH) void k_q4_read(const uint8_t *layer, T *__restrict__ k, T *__restrict__ v, int start, int rows, int tiles)
{
    using Tile = Q4Tile<DH>;
    constexpr int THREADS = 2 * DH, LANES = Tile::LANES, PASSES = FC_VTILE * LANES / THREADS, STEP = FC_VTILE / PASSES;
    __shared__ Tile s;
    const int tid = threadIdx.x, tile = start / FC_VTILE + blockIdx.x;
    const size_t pair = blockIdx.y;
    const uint8_t *rec = layer + (pair * tiles + tile) * (size_t)fc_q4_tile_bytes(DH);
    s.v[Tile::place(tid)] = ((const uint4 *)(rec + fc_q4_v(DH)))[tid];
    s.k[tid] = ((const uint4 *)rec)[tid];
    if (tid < Tile::SCALES / 4) ((uint32_t *)s.scale)[tid] = ((const uint32_t *)(rec + 64 * DH))[tid];
    __syncthreads();
    if (tid < DH) s.template turn<false>(tid);
    __syncthreads();
    const int lane = tid % LANES;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int r = tid / LANES + i * STEP, to = tile * FC_VTILE + r - start;
        if (to < 0 || to >= rows) continue;
        const size_t at = (pair * (size_t)rows + to) * DH + lane * 8;
        q4_put(k + at, s.key_word(r, lane), s.key_scale(r, lane / 4));
        q4_put(v + at, s.row[r * Tile::PITCH + lane], s.value_scale(r));
    }
}

template <typename T, int DH>
void launch_store(const FcQ4Geom &G, uint8_t *layer, const void *k, const void *v, const int32_t *pos, int start, int rows, int src_spad,
                  hipStream_t s)
{
    const int tiles = G.spad / FC_VTILE;
    const int n = pos ? (rows < tiles ? rows : tiles) : (start + rows - 1) / FC_VTILE - start / FC_VTILE + 1;
    const dim3 grid((unsigned)n, (unsigned)(G.B * G.Hkv));
    const Q4Place p{pos, start, rows, rows < tiles};
    if (src_spad)
        k_q4_store<T, DH, true, false><<<grid, dim3(2 * DH), 0, s>>>(layer, (const T *)k, (const T *)v, p, G.max_seq, tiles, src_spad, G.Hkv);
    else if (fc_read_once((double)G.B * G.Hkv * rows * (2.0 * DH * sizeof(T) + fc_q4_tile_bytes(DH) / 64)))  // (in and out)
        k_q4_store<T, DH, false, true><<<grid, dim3(2 * DH), 0, s>>>(layer, (const T *)k, (const T *)v, p, G.max_seq, tiles, rows, G.Hkv);
    else
        k_q4_store<T, DH, false, false><<<grid, dim3(2 * DH), 0, s>>>(layer, (const T *)k, (const T *)v, p, G.max_seq, tiles, rows, G.Hkv);
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
