// Bidirectional attention over a cache held in 4 bits (bf16 queries).
//
// S^T = K Q^T, softmax weights in registers, O^T = V^T W^T, one pass over the keys.  A wave holds 16 RT query rows (the rows of all
// query heads that share a kv head are one list) and takes tiles of 64 keys, straight from memory into operand registers: the
// tile's layout is the operands' (fc_q4.h), so the main loop has no barrier and, but for 64 scales, no lane crosses.
//
//  - Scores.  The 16x16x128 matrix instruction with block scales takes the key codes and their scales as they are stored; with a 6-bit other operand
//    it takes 16 clocks, a quarter of what bfloat16 products of that size take.  What a query lacks in bits it gets by parts: a lane's 32
//    elements of a row are three E2M3 numbers each, every one the rounding error of those before, 2^-16 of the largest of the 32 in the
//    end (the rows are bfloat16).  48 clocks, and no key is ever converted.  (Two e4m3 parts: 64 clocks.)
//  - Weights.  Value row t is codes times 2^e_t.  The power goes into the exponent of the row's weight, w_t = 2^(s_t + e_t - r), so the codes
//    are multiplied as they are, and the sum that divides adds w_t 2^-e_t.  The key multiply starts from e_t over the softmax scale, so this
//    costs nothing.  The reference r only has to keep w_t in range: it moves when a score passes it by 2^MOVE, which after the first
//    tiles is rare.  Weights are rounded to fp16 (11 bits; bfloat16 would add as much error as rounding the output does, two E2M3 parts
//    more, 2.8e-3 for 1.7e-3 relative in all), sums are fp32.
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
typedef float f16x __attribute__((ext_vector_type(16)));
typedef float f32x __attribute__((ext_vector_type(32)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef int i8x __attribute__((ext_vector_type(8)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u6 __attribute__((ext_vector_type(6)));

constexpr float MOVE = 8.f;  // a score may pass the reference by 2^MOVE

struct AttnArgs {
    const bf16_t *q;
    const uint8_t *layer;
    const int32_t *pos, *lens;
    bf16_t *out;
    float *part;  // partial results: [pair][split][rows][DH], then [pair][split][rows][2] (reference, sum)
    int A, kv_len, Hq, Hkv, g, tiles, rows, groups, splits, units;
    float c, by_c;  // scale * log2(e), and 1 / that
    FcDivisor by_groups, by_splits, by_hkv, by_a;
};

// What a wave loads of a tile.  Buffer loads: the place of the tile is a scalar, a lane keeps three offsets.
template <int DH>
struct Tile {
    u4 k[4], v[DH / 32];
    uint32_t ks, vs;
    __device__ __forceinline__ void load_keys(__amdgpu_buffer_rsrc_t r, uint32_t at, int lane)
    {
        const int kl = DH == 128 ? lane : lane & 31;  // (heads of 64: the upper lanes multiply the same keys with the second part)
#pragma unroll
        for (int t = 0; t < 4; ++t) k[t] = __builtin_amdgcn_raw_buffer_load_b128(r, kl * 16, at + t * (8 * DH), 0);
        ks = __builtin_amdgcn_raw_buffer_load_b32(r, kl * 4, at + 64 * DH, 0);
        vs = __builtin_amdgcn_raw_buffer_load_b32(r, lane & ~3, at + fc_q4_vscale(DH), 0);
    }
    __device__ __forceinline__ void load_values(__amdgpu_buffer_rsrc_t r, uint32_t at, int lane)
    {
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) v[j] = __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16, at + fc_q4_v(DH) + j * 1024, 0);
    }
};

// 32 values over `scale` as E2M3, and back.  The even ones come from `a`, the odd ones from `b`.  The instruction writes its first results before
// it has read its last sources and its scale: they are kept alive behind it, so that the compiler gives it other registers.
__device__ __forceinline__ u6 to_6bit(const f16x &a, const f16x &b, float scale)
{
    u6 c = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(a, b, scale);
    asm volatile("" : "+v"(c) : "v"(a), "v"(b), "v"(scale));
    return c;
}
// a, b less what `c` holds of them.
__device__ __forceinline__ void less_6bit(f16x &a, f16x &b, u6 c, float scale)
{
    f32x x = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(c, scale);
    asm volatile("" : "+v"(x) : "v"(c), "v"(scale));
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        a[i] -= x[2 * i];
        b[i] -= x[2 * i + 1];
    }
}
__device__ __forceinline__ i8x operand(const u4 &x) { return i8x{(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0}; }

// E2M1 codes times E2M3 ones; SA, SB: the byte of the scales' word.
template <int SA, int SB>
__device__ __forceinline__ f4 multiply(const i8x &codes, uint32_t sa, const i8x &part, uint32_t sb, f4 acc)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(codes, part, acc, 4, 2, SA, (int)sa, SB, (int)sb);
}

// Query rows as operands: N multiplies of a row tile, with the scales in one word.  Heads of 128: three parts, a multiply each.  Heads of 64: the
// first two parts are the two halves of one multiply (the lower lanes' keys against the first, the upper lanes' against the second), the
// third one half of another.
template <int DH, int RT>
struct Queries {
    static constexpr int N = DH == 128 ? 3 : 2;
    u4 lo[RT][N][64];
    u2 hi[RT][N][64];
    uint32_t scale[RT][64];

    __device__ __forceinline__ void fill(const bf16_t *q, int rt, int lane)  // q: the lane's 32 elements
    {
        u4 raw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = fc_load_any<u4>(q + i * 8);
        f16x a, b;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            a[i] = __uint_as_float(raw[i / 4][i % 4] << 16);
            b[i] = __uint_as_float(raw[i / 4][i % 4] & 0xffff0000u);
            top = max(top, max(__float_as_uint(a[i]) & 0x7fffffffu, __float_as_uint(b[i]) & 0x7fffffffu));
        }
        // the largest goes to 4 .. 7.5; below 2^-88 nothing need be exact
        const uint32_t e = max((top >> 23) + ((top & 0x7fffffu) > 0x700000u ? 1 : 0), 40u) - 2;
        u6 part[3];
        part[0] = to_6bit(a, b, __uint_as_float(e << 23));
        less_6bit(a, b, part[0], __uint_as_float(e << 23));
        part[1] = to_6bit(a, b, __uint_as_float((e - 4) << 23));  // (at most a quarter of a unit is left: 4 in units of 2^-4)
        less_6bit(a, b, part[1], __uint_as_float((e - 4) << 23));
        part[2] = to_6bit(a, b, __uint_as_float((e - 8) << 23));
        uint32_t s[3] = {e, e - 4, e - 8};
        if (top >= 0x7f800000u) s[0] = s[1] = s[2] = 255;  // not a number, and neither are the scores
        if constexpr (DH == 64) {
            const bool upper = lane >= 32;
            part[0] = upper ? part[1] : part[0];
            s[0] = upper ? s[1] : s[0];
            part[1] = upper ? u6{} : part[2];
            s[1] = s[2];
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            lo[rt][i][lane] = u4{part[i][0], part[i][1], part[i][2], part[i][3]};
            hi[rt][i][lane] = u2{part[i][4], part[i][5]};
        }
        scale[rt][lane] = s[0] | s[1] << 8 | s[2] << 16;
    }
    __device__ __forceinline__ i8x get(int rt, int i, int lane) const
    {
        const u4 x = lo[rt][i][lane];
        const u2 y = hi[rt][i][lane];
        return i8x{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], 0, 0};
    }
};

__device__ __forceinline__ float max16(const f4 (&s)[4])
{
    float m = fmaxf(s[0][0], s[0][1]);
#pragma unroll
    for (int i = 2; i < 16; i += 2) m = fmaxf(fmaxf(m, s[i / 4][i % 4]), s[i / 4][i % 4 + 1]);
    return m;
}

template <int DH, int RT, int W>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(2))) void k_q4_attn(AttnArgs p)
{
    constexpr int DT = DH / 16, N = Queries<DH, RT>::N;
    static_assert(RT <= W, "a wave converts one row tile at most");
    __shared__ f4 s_o[W][RT][DT][64];
    __shared__ Queries<DH, RT> s_q;
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

    f4 o[DT][RT];
    float ref[RT], sum[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        ref[rt] = -__builtin_inff();
        sum[rt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt][rt] = f4{0.f, 0.f, 0.f, 0.f};
    }
    Tile<DH> cur;
    int t = from + wave;
    if (t < to) {
        cur.load_keys(rsrc, (uint32_t)t * fc_q4_tile_bytes(DH), lane);
        cur.load_values(rsrc, (uint32_t)t * fc_q4_tile_bytes(DH), lane);
    }
    if (wave < RT) {
        const size_t row = min(row0 + wave * 16 + m, p.rows - 1);
        s_q.fill(p.q + (((size_t)b * p.Hq + (size_t)j * p.g) * p.A + row) * DH + (DH == 128 ? g : g & 1) * 32, wave, lane);
    }
    __syncthreads();
    i8x q[RT][N];
    uint32_t qs[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        qs[rt] = s_q.scale[rt][lane];
#pragma unroll
        for (int i = 0; i < N; ++i) q[rt][i] = s_q.get(rt, i, lane);
    }
    // The next tile's keys are loaded as soon as these are multiplied, its values likewise.  (Always, the last one once more: behind a
    // condition the compiler could not tell them from this tile's and would wait for them.)
    for (; t < to; t += W) {
        const uint32_t next = (uint32_t)min(t + W, to - 1) * fc_q4_tile_bytes(DH);
        // The row of this lane's scale byte: exponent / c, where the key multiply starts from, and 2^-exponent; then every lane takes those of
        // the sixteen rows whose weights it holds.
        {
            const float e = (float)max(cur.vs >> (lane % 4 * 8) & 255, (uint32_t)(FC_Q4_V_LOWEST + 127)) - 127.f;  // (a row never stored has 0)
            float start = e * p.by_c, f = __builtin_amdgcn_exp2f(-e);
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
// (part by part: products that add to one another are a latency of the matrix core apart)
#define FC_Q4_KEYS(T, I)                                                                    \
    _Pragma("unroll") for (int rt = 0; rt < RT; ++rt) s[rt][T] =                              \
        multiply<T, I>(operand(cur.k[T]), cur.ks, q[rt][I], qs[rt], I == 0 ? start[T] : s[rt][T]);
#define FC_Q4_PART(I) FC_Q4_KEYS(0, I) FC_Q4_KEYS(1, I) FC_Q4_KEYS(2, I) FC_Q4_KEYS(3, I)
        FC_Q4_PART(0)
        FC_Q4_PART(1)
        if constexpr (N == 3) { FC_Q4_PART(2) }
#undef FC_Q4_PART
#undef FC_Q4_KEYS
        cur.load_keys(rsrc, next, lane);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            top[rt] = max16(s[rt]) * p.c;
            move |= top[rt] > ref[rt] + MOVE;
        }
        if (__any(move)) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                float x = top[rt];
                x = fmaxf(x, __shfl_xor(x, 16));
                x = fmaxf(x, __shfl_xor(x, 32));
                const float r = fmaxf(ref[rt], x), a = __builtin_amdgcn_exp2f(ref[rt] - r);
                ref[rt] = r;
                sum[rt] *= a;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt][rt] *= a;
            }
        }
        h8 w[RT][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f4 f = *(const f4 *)&s_f[wave][g * 16 + i * 4];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(s[rt][i][k], p.c, -ref[rt]));
                    sum[rt] = fmaf(x, f[k], sum[rt]);
                    w[rt][i / 2][i % 2 * 4 + k] = (_Float16)x;
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
                for (int rt = 0; rt < RT; ++rt) o[dt][rt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w[rt][kb], o[dt][rt], 0, 0, 0);
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
        for (int dt = 0; dt < DT; ++dt) s_o[wave][rt][dt][lane] = o[dt][rt];
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
        const float inv = 1.f / l;
        bf16_t *out = p.out + ((size_t)b * p.A + a) * ((size_t)p.Hq * DH) + (size_t)(j * p.g + h) * DH + dt * 16 + g * 4;
        uint2 packed;
        packed.x = fc_bf16_bits(none ? 0.f : x[0] * inv) | (uint32_t)fc_bf16_bits(none ? 0.f : x[1] * inv) << 16;
        packed.y = fc_bf16_bits(none ? 0.f : x[2] * inv) | (uint32_t)fc_bf16_bits(none ? 0.f : x[3] * inv) << 16;
        fc_store_any(out, packed);
    }
}

// Partial results of the ranges, added at the largest reference; a thread has four elements of a row.  Eight ranges at a time, all their loads
// in flight together (one by one a range took 0.37 us).
template <int DH>
__global__ __launch_bounds__(256) void k_q4_merge(AttnArgs p)
{
    constexpr int T = DH / 4, N = 8;
    const uint32_t pair = blockIdx.y, b = p.by_hkv.over(pair), j = pair - b * p.Hkv;
    const int row = blockIdx.x * (256 / T) + threadIdx.x / T, d = threadIdx.x % T * 4;
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
    const float inv = 1.f / l;
    bf16_t *out = p.out + ((size_t)b * p.A + a) * ((size_t)p.Hq * DH) + (size_t)(j * p.g + h) * DH + d;
    uint2 packed;
    packed.x = fc_bf16_bits(none ? 0.f : x[0] * inv) | (uint32_t)fc_bf16_bits(none ? 0.f : x[1] * inv) << 16;
    packed.y = fc_bf16_bits(none ? 0.f : x[2] * inv) | (uint32_t)fc_bf16_bits(none ? 0.f : x[3] * inv) << 16;
    fc_store_any(out, packed);
}

template <int DH, int RT, int W>
void launch_w(const AttnArgs &p, hipStream_t s)
{
    const unsigned blocks = (unsigned)((p.units + 7) / 8 * 8 * p.groups);
    k_q4_attn<DH, RT, W><<<dim3(blocks), dim3(64 * W), 0, s>>>(p);
}
template <int DH>
void launch(const AttnArgs &p, const FcQ4Plan &pl, hipStream_t s)
{
    if (pl.rt == 2) pl.waves == 8 ? launch_w<DH, 2, 8>(p, s) : launch_w<DH, 2, 4>(p, s);
    else pl.waves == 8 ? launch_w<DH, 1, 8>(p, s) : launch_w<DH, 1, 4>(p, s);
    if (p.splits > 1) k_q4_merge<DH><<<dim3((unsigned)((p.rows + 1024 / DH - 1) / (1024 / DH)), (unsigned)(p.units / p.splits)), dim3(256), 0, s>>>(p);
}

// One wave per query row (fp32 queries), a key per lane for the scores and an element per lane for the sums: one pass over the keys with the running
// maximum and sum of the softmax.
template <typename T, int DH>
__global__ __launch_bounds__(64) void k_q4_rows(FcQ4Geom G, const T *__restrict__ q, const uint8_t *layer, const int32_t *__restrict__ pos,
                                                const int32_t *__restrict__ lens, int A, int kv_len, T *__restrict__ out)
{
    __shared__ float s_q[DH], s_p[64];
    const int lane = threadIdx.x, a = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    const int pair = b * G.Hkv + h / G.g;
    T *o = out + (((size_t)b * A + a) * G.Hq + h) * DH;
    const int n = lens ? min(max(lens[b], 0), kv_len) : kv_len;
    const bool empty = n == 0 || (pos && pos[(size_t)b * A + a] < 0);
    constexpr int E = DH / 64;
    float acc[E] = {}, top = -__builtin_inff(), sum = 0.f;
    if (!empty) {
        for (int i = lane; i < DH; i += 64) s_q[i] = fc_to_float(q[(((size_t)b * G.Hq + h) * A + a) * DH + i]) * G.scale;
        __syncthreads();
        for (int t0 = 0; t0 < n; t0 += FC_VTILE) {
            const uint8_t *rec = layer + ((size_t)pair * (G.spad / FC_VTILE) + t0 / FC_VTILE) * fc_q4_tile_bytes(DH);
            float s = 0.f;
            for (int c = 0; c < DH / 32; ++c) {
                const uint32_t *w = (const uint32_t *)(rec + fc_q4_k_block(DH, lane, c));
                float part = 0.f;
                for (int i = 0; i < 32; ++i) part += s_q[32 * c + i] * fc_q4_value(w[i / 8] >> (4 * (i % 8)) & 0xf);
                s += part * fc_q4_scale(rec[fc_q4_kscale(DH, lane, c)]);
            }
            if (t0 + lane >= n) s = -__builtin_inff();
            float m = s;
            for (int x = 1; x < 64; x <<= 1) m = fmaxf(m, __shfl_xor(m, x));
            const float next = fmaxf(top, m), old = expf(top - next), p = t0 + lane < n ? expf(s - next) : 0.f;
            float l = p;
            for (int x = 1; x < 64; x <<= 1) l += __shfl_xor(l, x);
            sum = sum * old + l;
            top = next;
            __syncthreads();
            s_p[lane] = t0 + lane < n ? p * fc_q4_scale(rec[fc_q4_vscale(DH) + fc_q4_vscale_at(lane)]) : 0.f;
            __syncthreads();
            const uint32_t *v = (const uint32_t *)(rec + fc_q4_v(DH));
            for (int e = 0; e < E; ++e) {
                const int d = 64 * e + lane;
                acc[e] *= old;
                for (int r0 = 0; r0 < 64; r0 += 32)
                    for (int g = 0; g < 4; ++g) {
                        const int w = d / 16 * 2 + r0 / 32;
                        const uint32_t code = v[w / 4 * 256 + (g * 16 + d % 16) * 4 + w % 4];
                        for (int j = 0; j < 8; ++j) acc[e] += s_p[r0 + j / 4 * 16 + g * 4 + j % 4] * fc_q4_value(code >> (4 * j) & 0xf);
                    }
            }
        }
    }
    for (int e = 0; e < E; ++e) o[64 * e + lane] = fc_from_float<T>(empty ? 0.f : acc[e] / sum);
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
const Q4Shape Q4_128[] = {{1, 4, 4.06, 0.650, 0.157, 0.65, 2.28, 0.077, 0.372, 0.59},
                          {1, 8, 3.47, 1.047, 0.158, 2.14, 2.10, 0.076, 0.434, 0.75},
                          {2, 4, 4.87, 0.920, 0.235, 1.43, 2.26, 0.087, 0.312, 0.70},
                          {2, 8, 4.11, 1.588, 0.244, 2.84, 2.19, 0.082, 0.386, 1.0}};
const Q4Shape Q4_64[] = {{1, 4, 3.77, 0.476, 0.098, 0.25, 2.13, 0.085, 0.404, 1.0},
                         {1, 8, 3.61, 0.757, 0.094, 0.74, 2.13, 0.082, 0.516, 0.65},
                         {2, 4, 4.49, 0.694, 0.161, 0.0, 2.05, 0.088, 0.606, 0.88},
                         {2, 8, 3.85, 1.161, 0.167, 0.98, 2.14, 0.066, 1.002, 0.92}};

// Estimated time of a call: the longest of a wave's chain of tiles, a compute unit's tiles and the stream from HBM, joined by a 4-norm, and the rest.
// The load of a compute unit is that of the die with the most units.  Fitted to 2344 measured (shape, plan) pairs of 110 shapes (1 .. 8 sequences, 1 ..
// 32 kv heads, 1 .. 8 query heads each, 1 .. 256 rows, 16 .. 16800 keys from HBM; rms error 4 .. 8 %); the plan it picks is 1.2 %
// slower than the best measured one in the mean, 13 % at most.
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
        best = FcQ4Plan{k.q4_rt == 2 ? 2 : 1, k.q4_waves == 8 ? 8 : 4, k.q4_splits > 0 ? k.q4_splits : 1};
        if (best.splits > tiles) best.splits = (int)tiles;
        while (best.splits > 1 && fc_q4_plan_workspace(G, best, A) > cap) --best.splits;
        return best;
    }
    double least = 1e30;
    for (const Q4Shape &sh : G.Dh == 128 ? Q4_128 : Q4_64) {
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
    if (G.dtype == FC_F32 || G.spad <= FC_VTILE) return 0;
    const int64_t rows = (int64_t)G.B * G.Hkv * G.g * max_rows * MOST_SPLITS, most = (int64_t)MOST_WGS * 32;
    return (size_t)(rows < most ? rows : most) * (G.Dh + 2) * sizeof(float);
}

FcQ4Plan fc_plan_q4(const FcQ4Geom &G, int A, int kv_len, size_t cap)
{
    if (G.dtype == FC_F32) return FcQ4Plan{1, 4, 1};
    const size_t most = fc_q4_most_workspace(G, A);
    if (cap > most && !fc_knobs().q4_rt) cap = most;  // (more changes nothing)
    // The last few plans of this thread: a program calls with one shape for every layer.
    struct Entry {
        int key[7];
        size_t cap;
        FcQ4Plan plan;
    };
    static thread_local Entry known[4];
    static thread_local unsigned next = 0;
    const int key[7] = {G.B, G.Hkv, G.g, G.Dh, A, kv_len, fc_knobs().version + 1};
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
    if (G.dtype == FC_F32) {
        const dim3 grid((unsigned)A, (unsigned)G.Hq, (unsigned)G.B);
        if (G.Dh == 128) k_q4_rows<float, 128><<<grid, dim3(64), 0, s>>>(G, (const float *)q, layer, pos, lens, A, kv_len, (float *)out);
        else k_q4_rows<float, 64><<<grid, dim3(64), 0, s>>>(G, (const float *)q, layer, pos, lens, A, kv_len, (float *)out);
        return hipGetLastError();
    }
    AttnArgs p;
    p.q = (const bf16_t *)q;
    p.layer = layer;
    p.pos = pos;
    p.lens = lens;
    p.out = (bf16_t *)out;
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
    if (G.Dh == 128) launch<128>(p, pl, s);
    else launch<64>(p, pl, s);
    return hipGetLastError();
}
