// Bidirectional attention over a cache held in 4 bits.
//
// S^T = K Q^T, softmax weights in registers, O^T = V^T W^T, one pass over the keys.  A wave holds 16 RT query rows (the rows of all
// query heads that share a kv head are one list) and takes tiles of 64 keys, straight from memory into operand registers: the
// tile's layout is the operands' (fc_q4.h), so the main loop has no barrier and, but for 64 scales, no lane crosses.
//
//  - Scores.  Key codes become bfloat16 by one conversion for two (a number of the format times its power of two is one, exactly), once for all
//    RT row tiles, and a bfloat16 row is multiplied as it is: nothing is lost before the sums in fp32, however far the elements of a row
//    are apart.  (The matrix instructions with block scales take the codes unconverted, but the row then has to go in as 6-bit numbers,
//    each part 5 bits more below the largest of 32 elements: with three parts, 2^-14, channels 256 times the others cost 3.5e-3 of
//    the result, and four take as long as the conversions.  As two 8-bit numbers its products would be cut off at 2^-14 of their sum.)
//  - Weights.  Value row t is codes times 2^e_t.  The power goes into the exponent of the row's weight, w_t = 2^(s_t + e_t - r), so the codes
//    are multiplied as they are, and the sum that divides adds w_t 2^-e_t.  The key multiply starts from e_t over the softmax scale, so this
//    costs nothing.  The reference r only has to keep w_t in range: it is set 2^7 below the largest and moves when a score passes it by 2^14, which after
//    the first tiles is rare.  Weights are rounded to fp16: 11 bits down to 2^-21 of the largest, none below 2^-32 (half a step of the least
//    number; the sum that divides has them all, in fp32).  bfloat16 would add as much error as rounding the output does, two E2M3 parts
//    more, 2.8e-3 for 1.7e-3 relative in all.  Sums are fp32.
//  - fp32 rows are three bfloat16 numbers, 8 bits each, which is all of them, and a weight is two fp16 numbers, the second in units of 2^-12 with sums
//    of its own: 2^-23 of the weight.  The reference is a whole number and e_t - r is added with the scale, so a score is rounded once.
//    Errors against 64 bits are 1.6e-7 (heads of 64) and 2.2e-7 (128), less than half of a plain fp32 computation's; 32 rows x 28 heads over
//    1056 keys take 9.9 us (bfloat16: 6.8).
//  - Values.  Codes become fp16 pairs by one conversion each, once for all RT row tiles.
//
// The waves of a workgroup take tiles in turn and add up in LDS at the end.  Where there are few (sequence, kv head, row group)
// units, the tiles are cut into ranges, and a second kernel adds their partial results, in fp32.
#include <math.h>
#include <string.h>

#include "fc_device.h"
#include "fc_internal.h"
#include "fc_q4.h"

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr float LIFT = 7.f;   // a row's largest weight so far is 2^LIFT when its reference is set
constexpr float MOVE = 14.f;  // and none may pass 2^MOVE but for roundings: fp16 ends at 65504 (fp32: half its step there, 8, times FINE does too)
constexpr float HUGE_REF = 0x1p20f;  // from here on the roundings of a score decide weights
constexpr float FINE = 4096.f;  // fp32: what a weight's fp16 lacks is multiplied in units of 1 / FINE
template <typename T> constexpr int MOST_RT = sizeof(T) == 4 ? 1 : 2;  // row tiles of a workgroup

struct AttnArgs {
    const void *q;
    const uint8_t *layer;
    const int32_t *pos, *lens;
    void *out;
    float *part;  // partial results: [pair][split][rows][DH], then [pair][split][rows][2] (reference, sum)
    int A, kv_len, Hq, Hkv, g, tiles, rows, groups, splits, units;
    float c, by_c;  // scale * log2(e), and 1 / that
    FcDivisor by_groups, by_splits, by_hkv, by_a;
};

// What a wave loads of a tile.  Buffer loads: the place of the tile is a scalar, a lane keeps three offsets.
template <int DH>
struct Tile {
    uint32_t k[4][DH / 32];
    u4 v[DH / 32];
    uint32_t ks, vs;
    __device__ __forceinline__ void load_keys(__amdgpu_buffer_rsrc_t r, uint32_t at, int lane)
    {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if constexpr (DH == 128) {
                const u4 x = __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16, at + t * (8 * DH), 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) k[t][i] = x[i];
            } else {  // (two blocks to a row: the upper lanes have the second half of the lower ones')
                const u2 x = __builtin_amdgcn_raw_buffer_load_b64(r, (lane & 31) * 16 + (lane >> 5) * 8, at + t * (8 * DH), 0);
                k[t][0] = x[0];
                k[t][1] = x[1];
            }
        }
        ks = __builtin_amdgcn_raw_buffer_load_b32(r, (DH == 128 ? lane : lane & 31) * 4, at + 64 * DH, 0);
        vs = __builtin_amdgcn_raw_buffer_load_b32(r, lane & ~3, at + fc_q4_vscale(DH), 0);
    }
    __device__ __forceinline__ void load_values(__amdgpu_buffer_rsrc_t r, uint32_t at, int lane)
    {
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) v[j] = __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16, at + fc_q4_v(DH) + j * 1024, 0);
    }
};

// Eight key codes as bfloat16.
__device__ __forceinline__ b8 key_values(uint32_t c, float scale)
{
    struct {
        b2 v[4];
    } x = {{__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((int)c, scale, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((int)c, scale, 1),
            __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((int)c, scale, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((int)c, scale, 3)}};
    return __builtin_bit_cast(b8, x);
}

// Query rows of a wave as operands: PARTS of bfloat16, N multiplies each.  A lane has the elements that its key codes are multiplied by: those of block
// lane / 16, or (heads of 64) half a block.
template <typename T, int DH, int RT>
struct Queries {
    static constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, N = DH / 32;
    b8 x[RT][PARTS][N];
    static __device__ __forceinline__ int first(int lane) { return DH == 128 ? lane / 16 * 32 : (lane / 16 & 1) * 32 + lane / 32 * 16; }
    __device__ __forceinline__ void load(const bf16_t *q, int rt)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) x[rt][0][i] = __builtin_bit_cast(b8, fc_load_any<u4>(q + i * 8));
    }
    __device__ __forceinline__ void load(const float *q, int rt)
    {
        struct {
            f4 v[2 * N];
        } raw;
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) raw.v[i] = fc_load_any<f4>(q + i * 4);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t word[PARTS][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float a = raw.v[2 * i + j / 2][j % 2 * 2], b = raw.v[2 * i + j / 2][j % 2 * 2 + 1];
#pragma unroll
                for (int k = 0; k < PARTS; ++k) {  // the upper 16 bits; what they leave is exact, and after three parts nothing
                    const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
                    word[k][j] = __builtin_amdgcn_perm(ub, ua, 0x07060302);
                    a -= __uint_as_float(ua & 0xffff0000u);
                    b -= __uint_as_float(ub & 0xffff0000u);
                }
            }
#pragma unroll
            for (int k = 0; k < PARTS; ++k) x[rt][k][i] = __builtin_bit_cast(b8, word[k]);
        }
    }
};

__device__ __forceinline__ float max16(const f4 (&s)[4])
{
    float m = fmaxf(s[0][0], s[0][1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) m = fmaxf(fmaxf(m, s[i / 4][i % 4]), s[i / 4][i % 4 + 1]);
    return m;
}

// Four elements of a result.
__device__ __forceinline__ void put(bf16_t *to, const f4 &x)
{
    fc_store_any(to, uint2{fc_bf16_bits(x[0]) | (uint32_t)fc_bf16_bits(x[1]) << 16, fc_bf16_bits(x[2]) | (uint32_t)fc_bf16_bits(x[3]) << 16});
}
__device__ __forceinline__ void put(float *to, const f4 &x) { fc_store_any(to, x); }

template <typename T, int DH, int RT, int W>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(2))) void k_q4_attn(AttnArgs p)
{
    constexpr bool FULL = sizeof(T) == 4;
    using Q = Queries<T, DH, RT>;
    constexpr int DT = DH / 16;
    __shared__ f4 s_o[W][RT][DT][64];
    __shared__ float s_ref[W][RT * 16], s_sum[W][RT * 16];
    __shared__ __align__(16) float s_start[W][64], s_f[W][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = lane % 16, g = lane / 16;
    // Workgroups go to the eight dies in turn: those of one unit (a range of one sequence and kv head) get places 8 apart, so that its row
    // groups read the tiles through one L2.
    const uint32_t slot = blockIdx.x >> 3, turn = p.by_groups.over(slot), group = slot - turn * p.groups, unit = turn * 8 + (blockIdx.x & 7);
    if (unit >= (uint32_t)p.units) return;
    const uint32_t pair = p.by_splits.over(unit), split = unit - pair * p.splits;
    const uint32_t b = p.by_hkv.over(pair), j = pair - b * p.Hkv;
    const int n = p.lens ? min(max(p.lens[b], 0), p.kv_len) : p.kv_len;
    const int row0 = (int)group * RT * 16;
    const int all = (n + 63) / 64, per = (int)p.by_splits.over((uint32_t)(all + p.splits - 1));
    const int from = min(all, (int)split * per), to = min(all, from + per);
    // (at most 2^18 tiles: offsets fit 32 bits)
    const uint32_t bytes = (uint32_t)p.tiles * fc_q4_tile_bytes(DH);
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(p.layer + (size_t)pair * bytes), 0, (int)bytes, 0x00020000);

    f4 o[DT][RT], fine[FULL ? DT : 1][RT];
    float ref[RT], sum[RT];
    bool huge = false;  // a reference whose roundings count
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        ref[rt] = -__builtin_inff();
        sum[rt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt][rt] = fine[FULL ? dt : 0][rt] = f4{0.f, 0.f, 0.f, 0.f};
    }
    Tile<DH> cur;
    int t = from + wave;
    if (t < to) {
        cur.load_keys(rsrc, (uint32_t)t * fc_q4_tile_bytes(DH), lane);
        cur.load_values(rsrc, (uint32_t)t * fc_q4_tile_bytes(DH), lane);
    }
    Q q;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const size_t row = min(row0 + rt * 16 + m, p.rows - 1);
        q.load((const T *)p.q + (((size_t)b * p.Hq + (size_t)j * p.g) * p.A + row) * DH + Q::first(lane), rt);
    }
    // The next tile's keys are loaded as soon as these are multiplied, its values likewise.  (Always, the last one once more: behind a
    // condition the compiler could not tell them from this tile's and would wait for them.)
    for (; t < to; t += W) {
        const uint32_t next = (uint32_t)min(t + W, to - 1) * fc_q4_tile_bytes(DH);
        // The row of this lane's scale byte: exponent / c, where the key multiply starts from, and 2^-exponent; then every lane takes those of
        // the sixteen rows whose weights it holds.
        {
            const uint32_t byte = cur.vs >> (lane % 4 * 8) & 255;
            const float e = (float)max(byte, (uint32_t)(FC_Q4_V_LOWEST + 127)) - 127.f;  // (a row never stored has 0)
            float start = byte == 255 ? __builtin_nanf("") : FULL ? e : e * p.by_c, f = __builtin_amdgcn_exp2f(-e);
            if ((t + 1) * 64 > n) {  // rows behind the end may hold anything: weight 0, and key scales that leave scores finite
                if (t * 64 + lane % 16 / 4 * 16 + g * 4 + lane % 4 >= n) {
                    start = -__builtin_inff();
                    f = 0.f;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (t * 64 + i * 16 + m >= n) cur.ks &= ~(0xffu << (8 * i));
            }
            s_start[wave][lane] = start;
            s_f[wave][lane] = f;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        f4 start[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) start[i] = *(const f4 *)&s_start[wave][g * 16 + i * 4];
        f4 s[RT][4];
        bool move = false;
        float top[RT];
        // (the least part first; products that add to one another are a latency of the matrix core apart)
#pragma unroll
        for (int i = 0; i < Q::N; ++i) {
            b8 keys[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) keys[k] = key_values(cur.k[k][i], __uint_as_float((cur.ks >> (8 * k) & 255) << 23));
#pragma unroll
            for (int part = Q::PARTS - 1; part >= 0; --part)
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        const f4 sum = i || part + 1 < Q::PARTS ? s[rt][k] : FULL ? f4{0.f, 0.f, 0.f, 0.f} : start[k];
                        s[rt][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(keys[k], q.x[rt][part][i], sum, 0, 0, 0);
                    }
        }
        cur.load_keys(rsrc, next, lane);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if constexpr (FULL) {
                f4 x[4];
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i / 4][i % 4] = fmaf(s[rt][i / 4][i % 4], p.c, start[i / 4][i % 4]);
                top[rt] = max16(x);
            } else {
                top[rt] = max16(s[rt]) * p.c;
            }
            move |= top[rt] - ref[rt] > MOVE;
        }
        if (__any(move)) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                float x = top[rt];
                x = fmaxf(x, __shfl_xor(x, 16));
                x = fmaxf(x, __shfl_xor(x, 32));
                const float r = fmaxf(ref[rt], (FULL ? ceilf(x) : x) - LIFT), a = __builtin_amdgcn_exp2f(ref[rt] - r);
                ref[rt] = r;
                sum[rt] *= a;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    o[dt][rt] *= a;
                    if constexpr (FULL) fine[dt][rt] *= a;
                }
                huge |= __any(fabsf(r) > HUGE_REF && fabsf(r) < __builtin_inff());  // (rows that are not numbers change no other's bits)
            }
        }
        // A weight's exponent.  Where the scores are so large that the product with the scale is off by what decides a weight, it is rounded as the
        // largest's was, which the reference comes from: none then passes that one, and the largest is not lost.
        if (__builtin_expect(!huge, 1)) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[rt][i / 4][i % 4] = fmaf(s[rt][i / 4][i % 4], p.c, FULL ? start[i / 4][i % 4] - ref[rt] : -ref[rt]);
        } else {
#pragma clang fp contract(off)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = FULL ? fmaf(s[rt][i / 4][i % 4], p.c, start[i / 4][i % 4]) : s[rt][i / 4][i % 4] * p.c;
                    s[rt][i / 4][i % 4] = x - ref[rt];
                }
        }
        h8 w[RT][2], rest[RT][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f4 f = *(const f4 *)&s_f[wave][g * 16 + i * 4];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float x = __builtin_amdgcn_exp2f(s[rt][i][k]);
                    sum[rt] = fmaf(x, f[k], sum[rt]);
                    w[rt][i / 2][i % 2 * 4 + k] = (_Float16)x;
                    if constexpr (FULL) rest[rt][i / 2][i % 2 * 4 + k] = (_Float16)((x - (float)(_Float16)x) * FINE);
                }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const uint32_t c = cur.v[dt / 2][dt % 2 * 2 + kb];
                h8 v;
#define FC_Q4_VALUES(B)                                                             \
    {                                                                               \
        const h2 x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4((int)c, 1.0f, B);     \
        v[2 * B] = x[0];                                                            \
        v[2 * B + 1] = x[1];                                                        \
    }
                FC_Q4_VALUES(0)
                FC_Q4_VALUES(1)
                FC_Q4_VALUES(2)
                FC_Q4_VALUES(3)
#undef FC_Q4_VALUES
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    o[dt][rt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w[rt][kb], o[dt][rt], 0, 0, 0);
                    if constexpr (FULL) fine[dt][rt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, rest[rt][kb], fine[dt][rt], 0, 0, 0);
                }
            }
        cur.load_values(rsrc, next, lane);
    }

    // The waves' results: every one at the largest reference, added by pieces of 16 rows x 16 elements.
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float l = sum[rt];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (g == 0) {
            s_ref[wave][rt * 16 + m] = ref[rt];
            s_sum[wave][rt * 16 + m] = l;
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) s_o[wave][rt][dt][lane] = FULL ? o[dt][rt] + fine[FULL ? dt : 0][rt] * (1.f / FINE) : o[dt][rt];
    }
    __syncthreads();
#pragma unroll 1
    for (int piece = wave; piece < RT * DT; piece += W) {
        const int rt = piece / DT, dt = piece % DT, row = row0 + rt * 16 + m;
        if (row >= p.rows) continue;
        float top = s_ref[0][rt * 16 + m], l = 0.f;
#pragma unroll
        for (int i = 1; i < W; ++i) top = fmaxf(top, s_ref[i][rt * 16 + m]);
        f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float a = from + i < to ? __builtin_amdgcn_exp2f(s_ref[i][rt * 16 + m] - top) : 0.f;
            l = fmaf(a, s_sum[i][rt * 16 + m], l);
            x += a * s_o[i][rt][dt][lane];
        }
        if (p.splits > 1) {
            const size_t at = (size_t)unit * p.rows + row;
            *(f4 *)(p.part + at * DH + dt * 16 + g * 4) = x;
            if (dt == 0 && g == 0) {
                float *st = p.part + (size_t)p.units * p.rows * DH + at * 2;
                st[0] = top;
                st[1] = l;
            }
            continue;
        }
        const uint32_t h = p.by_a.over(row), a = row - h * p.A;
        const bool none = n == 0 || (p.pos && p.pos[(size_t)b * p.A + a] < 0);
        T *out = (T *)p.out + ((size_t)b * p.A + a) * ((size_t)p.Hq * DH) + (size_t)(j * p.g + h) * DH + dt * 16 + g * 4;
        put(out, none ? f4{0.f, 0.f, 0.f, 0.f} : x * (1.f / l));
    }
}

// Partial results of the ranges, added at the largest reference; a thread has four elements of a row.  Eight ranges at a time, all their loads
// in flight together (one by one a range took 0.37 us).
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_q4_merge(AttnArgs p)
{
    constexpr int LANES = DH / 4, N = 8;
    const uint32_t pair = blockIdx.y, b = p.by_hkv.over(pair), j = pair - b * p.Hkv;
    const int row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, d = threadIdx.x % LANES * 4;
    if (row >= p.rows) return;
    const float2 *st = (const float2 *)(p.part + (size_t)p.units * p.rows * DH);
    const size_t at = (size_t)pair * p.splits * p.rows + row;
    const uint32_t h = p.by_a.over(row), a = row - h * p.A;
    const int n = p.lens ? min(max(p.lens[b], 0), p.kv_len) : p.kv_len;
    const bool none = n == 0 || (p.pos && p.pos[(size_t)b * p.A + a] < 0);
    const int all = (n + 63) / 64, per = max((int)p.by_splits.over((uint32_t)(all + p.splits - 1)), 1);
    const int used = (all + per - 1) / per;  // (of a short sequence the last ranges are empty)
    float top = -__builtin_inff(), l = 0.f;
    f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int s0 = 0; s0 < used; s0 += N) {
        float2 state[N];
        f4 v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const size_t k = at + (size_t)min(s0 + i, used - 1) * p.rows;
            state[i] = st[k];
            v[i] = *(const f4 *)(p.part + k * DH + d);
        }
        __builtin_amdgcn_sched_barrier(0);
        float next = top;
#pragma unroll
        for (int i = 0; i < N; ++i) next = fmaxf(next, state[i].x);
        const float old = s0 ? __builtin_amdgcn_exp2f(top - next) : 0.f;
        l *= old;
        x *= old;
        top = next;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (s0 + i >= used) continue;
            const float w = __builtin_amdgcn_exp2f(state[i].x - top);
            l = fmaf(w, state[i].y, l);
            x += w * v[i];
        }
    }
    T *out = (T *)p.out + ((size_t)b * p.A + a) * ((size_t)p.Hq * DH) + (size_t)(j * p.g + h) * DH + d;
    put(out, none ? f4{0.f, 0.f, 0.f, 0.f} : x * (1.f / l));
}

template <typename T, int DH, int RT, int W>
void launch_w(const AttnArgs &p, hipStream_t s)
{
    const unsigned blocks = (unsigned)((p.units + 7) / 8 * 8 * p.groups);
    k_q4_attn<T, DH, RT, W><<<dim3(blocks), dim3(64 * W), 0, s>>>(p);
}
template <typename T, int DH>
void launch(const AttnArgs &p, const FcQ4Plan &pl, hipStream_t s)
{
    constexpr int RT = MOST_RT<T>;
    if (pl.rt == 2) pl.waves == 8 ? launch_w<T, DH, RT, 8>(p, s) : launch_w<T, DH, RT, 4>(p, s);
    else if (pl.waves > 2) pl.waves == 8 ? launch_w<T, DH, 1, 8>(p, s) : launch_w<T, DH, 1, 4>(p, s);
    else pl.waves == 2 ? launch_w<T, DH, 1, 2>(p, s) : launch_w<T, DH, 1, 1>(p, s);
    if (p.splits > 1) k_q4_merge<T, DH><<<dim3((unsigned)((p.rows + 1024 / DH - 1) / (1024 / DH)), (unsigned)(p.units / p.splits)), dim3(256), 0, s>>>(p);
}

}  // namespace

size_t fc_q4_plan_workspace(const FcQ4Geom &G, const FcQ4Plan &pl, int A)
{
    return pl.splits > 1 ? (size_t)G.B * G.Hkv * pl.splits * G.g * A * (G.Dh + 2) * sizeof(float) : 0;
}

namespace {

constexpr int MOST_SPLITS = 64, MOST_WGS = 512;  // of a call that cuts the keys (more never came out best)
const int SPLITS[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64};

// What a workgroup shape takes (us): start and end; a tile of a wave; a tile of a compute unit, its loads and multiplies; a workgroup of a compute
// unit; a second kernel, each range of it, and a MB of partial results.  `part`: what a last partly filled round costs at least.
struct Q4Shape {
    int rt, waves;
    double start, wave, unit, wg, merge, range, mb, part;
};
const Q4Shape Q4_128[] = {{1, 1, 3.85, 0.716, 0.193, 0.29, 1.71, 0.079, 0.353, 0.98},
                          {1, 2, 3.25, 0.766, 0.217, 0.39, 2.07, 0.081, 0.367, 1.00},
                          {1, 4, 3.06, 0.777, 0.175, 0.69, 2.19, 0.079, 0.345, 0.68},
                          {1, 8, 2.47, 1.270, 0.195, 1.79, 2.21, 0.083, 0.295, 0.72},
                          {2, 4, 3.93, 1.096, 0.275, 1.43, 2.29, 0.063, 0.331, 0.56},
                          {2, 8, 3.11, 1.933, 0.331, 2.82, 2.39, 0.052, 0.320, 0.60}};
const Q4Shape Q4_64[] = {{1, 1, 3.09, 0.557, 0.134, 0.12, 1.83, 0.073, 0.554, 1.00},
                         {1, 2, 2.85, 0.603, 0.117, 0.22, 2.02, 0.070, 0.633, 1.00},
                         {1, 4, 2.76, 0.599, 0.107, 0.31, 2.09, 0.067, 0.515, 1.00},
                         {1, 8, 2.70, 0.868, 0.107, 0.72, 2.06, 0.059, 0.452, 0.66},
                         {2, 4, 3.40, 0.829, 0.173, 0.64, 2.02, 0.054, 0.573, 0.70},
                         {2, 8, 2.72, 1.348, 0.213, 1.51, 2.04, 0.036, 0.694, 0.92}};
const Q4Shape Q4_F32_128[] = {{1, 1, 4.35, 1.166, 0.306, 0.55, 1.83, 0.087, 0.311, 0.06},
                              {1, 2, 3.91, 1.179, 0.474, 0.56, 2.18, 0.094, 0.215, 1.00},
                              {1, 4, 3.68, 1.244, 0.363, 1.22, 2.26, 0.090, 0.247, 0.40},
                              {1, 8, 2.61, 2.277, 0.489, 2.31, 2.27, 0.086, 0.297, 0.62}};
const Q4Shape Q4_F32_64[] = {{1, 1, 3.43, 0.801, 0.226, 0.20, 2.13, 0.059, 0.362, 0.22},
                             {1, 2, 3.30, 0.805, 0.316, 0.09, 2.24, 0.076, 0.269, 1.00},
                             {1, 4, 3.13, 0.819, 0.229, 0.38, 2.38, 0.044, 0.419, 0.60},
                             {1, 8, 2.93, 1.347, 0.274, 1.25, 2.29, 0.000, 0.754, 0.59}};

// Estimated time of a call: the longest of a wave's chain of tiles, a compute unit's tiles and the stream from HBM, joined by a 4-norm, and the rest.
// The load of a compute unit is that of the die with the most units.  Fitted to 3804 measured (shape, plan) pairs of 160 shapes in bf16 and 1744 of 80 in
// fp32 (1 .. 8 sequences, 1 .. 32 kv heads, 1 .. 8 query heads each, 1 .. 256 rows, 8 .. 16800 keys from HBM; rms error of a shape
// 5 .. 10 %); the plan it picks is 1.6 % (fp32: 2.7) slower than the best measured one in the mean, 11 % (17) at most.  fp32 has tables of its
// own: by bf16's it came out 3.4 % slower in the mean, 34 at most, as a tile takes it twice as long.  One wave is for few keys and many
// rows: 4 sequences, 8 kv heads of 7, 160 rows, 32 keys take 8.7 us with one, 11.5 with four; 8 sequences, 28 / 4 heads, 256 rows, 128
// keys 14.9 and 19.0.
double q4_cost(const Q4Shape &sh, int64_t pairs, int64_t rows, int64_t tiles, int dh, int64_t splits)
{
    const int64_t groups = (rows + 16 * sh.rt - 1) / (16 * sh.rt), per = (tiles + splits - 1) / splits;
    double load = (double)((pairs * splits + 7) / 8 * groups) / 32.0;
    if (load > 1.0) {
        const double whole = floor(load);
        if (load > whole) load = whole + sh.part + (1.0 - sh.part) * (load - whole);
    }
    const double wave = sh.wave * (double)((per + sh.waves - 1) / sh.waves), unit = sh.unit * load * (double)per;
    const double hbm = (double)pairs * (double)tiles * (66.0 * dh + 64.0) / 5.5e6;
    const double w2 = wave * wave, u2 = unit * unit, h2 = hbm * hbm;
    double us = sh.start + sqrt(sqrt(w2 * w2 + u2 * u2 + h2 * h2)) + sh.wg * load;
    if (splits > 1) us += sh.merge + sh.range * (double)splits + sh.mb * (double)(pairs * rows * splits * dh) * 4e-6;
    return us;
}

FcQ4Plan plan(const FcQ4Geom &G, int A, int kv_len, size_t cap)
{
    const int64_t pairs = (int64_t)G.B * G.Hkv, rows = (int64_t)G.g * A, tiles = ((int64_t)kv_len + FC_VTILE - 1) / FC_VTILE;
    FcQ4Plan best{1, 4, 1};
    const FcKnobs &k = fc_knobs();
    if (k.q4_rt > 0) {  // a tuning knob asks for one
        best.rt = k.q4_rt == 2 && G.dtype != FC_F32 ? 2 : 1;
        best.waves = k.q4_waves == 8 || (best.rt == 1 && (k.q4_waves == 1 || k.q4_waves == 2)) ? k.q4_waves : 4;
        best.splits = k.q4_splits > 0 ? k.q4_splits : 1;
        if (best.splits > tiles) best.splits = (int)tiles;
        const int64_t groups = (rows + 16 * best.rt - 1) / (16 * best.rt);
        while (best.splits > 1 && (fc_q4_plan_workspace(G, best, A) > cap || (pairs * best.splits + 7) * groups >= 1 << 23)) --best.splits;
        return best;
    }
    double least = 1e30;
    const bool f32 = G.dtype == FC_F32;
    const Q4Shape *const shapes = f32 ? (G.Dh == 128 ? Q4_F32_128 : Q4_F32_64) : G.Dh == 128 ? Q4_128 : Q4_64;
    for (int i = 0; i < (f32 ? 4 : 6); ++i) {
        const Q4Shape &sh = shapes[i];
        const int64_t groups = (rows + 16 * sh.rt - 1) / (16 * sh.rt);
        for (const int splits : SPLITS) {
            const FcQ4Plan pl{sh.rt, sh.waves, splits};
            if (splits > 1 && (splits > tiles || pairs * groups * splits > MOST_WGS || fc_q4_plan_workspace(G, pl, A) > cap)) break;
            const double us = q4_cost(sh, pairs, rows, tiles, G.Dh, splits);
            if (us < least) {
                least = us;
                best = pl;
            }
        }
    }
    return best;
}

}  // namespace

// Upper bound of what a plan for up to max_rows rows uses: 64 ranges of every row, or 512 workgroups of 32 rows.
size_t fc_q4_most_workspace(const FcQ4Geom &G, int max_rows)
{
    if (G.spad <= FC_VTILE) return 0;
    const int64_t rows = (int64_t)G.B * G.Hkv * G.g * max_rows * MOST_SPLITS, most = (int64_t)MOST_WGS * 32;
    return (size_t)(rows < most ? rows : most) * (G.Dh + 2) * sizeof(float);
}

FcQ4Plan fc_plan_q4(const FcQ4Geom &G, int A, int kv_len, size_t cap)
{
    const size_t most = fc_q4_most_workspace(G, A);
    if (cap > most && !fc_knobs().q4_rt) cap = most;  // (more changes nothing)
    // The last few plans of this thread: a program calls with one shape for every layer.
    struct Entry {
        int key[8];
        size_t cap;
        FcQ4Plan plan;
    };
    static thread_local Entry known[4];
    static thread_local unsigned next = 0;
    const int key[8] = {G.B, G.Hkv, G.g, G.Dh, G.dtype, A, kv_len, fc_knobs().version + 1};
    for (const Entry &e : known)
        if (e.cap == cap && !memcmp(e.key, key, sizeof key)) return e.plan;
    Entry &e = known[next++ % 4];
    memcpy(e.key, key, sizeof key);
    e.cap = cap;
    return e.plan = plan(G, A, kv_len, cap);
}

hipError_t fc_launch_q4_attention(const FcQ4Geom &G, const FcQ4Plan &pl, const void *q, const uint8_t *layer, const int32_t *pos, const int32_t *lens,
                                  int A, int kv_len, void *out, void *workspace, hipStream_t s)
{
    AttnArgs p;
    p.q = q;
    p.layer = layer;
    p.pos = pos;
    p.lens = lens;
    p.out = out;
    p.part = (float *)workspace;
    p.A = A;
    p.kv_len = kv_len;
    p.Hq = G.Hq;
    p.Hkv = G.Hkv;
    p.g = G.g;
    p.tiles = G.spad / FC_VTILE;
    p.rows = G.g * A;
    p.groups = (p.rows + 16 * pl.rt - 1) / (16 * pl.rt);
    p.splits = pl.splits;
    p.units = G.B * G.Hkv * pl.splits;
    p.c = G.scale * 1.4426950408889634f;
    p.by_c = 1.f / p.c;
    p.by_groups.set((uint32_t)p.groups);
    p.by_splits.set((uint32_t)p.splits);
    p.by_hkv.set((uint32_t)p.Hkv);
    p.by_a.set((uint32_t)A);
    if (G.dtype == FC_F32) G.Dh == 128 ? launch<float, 128>(p, pl, s) : launch<float, 64>(p, pl, s);
    else G.Dh == 128 ? launch<bf16_t, 128>(p, pl, s) : launch<bf16_t, 64>(p, pl, s);
    return hipGetLastError();
}
