// Bidirectional attention over a cache held in 4 bits.
#include "fc_device.h"
#include "fc_internal.h"
#include "fc_q4.h"

namespace {

// One wave per query row, a key per lane for the scores and an element per lane for the sums: one pass over the keys with the running
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

hipError_t fc_launch_q4_attention(const FcQ4Geom &G, const void *q, const uint8_t *layer, const int32_t *pos, const int32_t *lens, int A, int kv_len,
                                  void *out, void *workspace, hipStream_t s)
{
    const dim3 grid((unsigned)A, (unsigned)G.Hq, (unsigned)G.B);
    if (G.dtype == FC_F32) {
        if (G.Dh == 128) k_q4_rows<float, 128><<<grid, dim3(64), 0, s>>>(G, (const float *)q, layer, pos, lens, A, kv_len, (float *)out);
        else k_q4_rows<float, 64><<<grid, dim3(64), 0, s>>>(G, (const float *)q, layer, pos, lens, A, kv_len, (float *)out);
    } else {
        if (G.Dh == 128) k_q4_rows<bf16_t, 128><<<grid, dim3(64), 0, s>>>(G, (const bf16_t *)q, layer, pos, lens, A, kv_len, (bf16_t *)out);
        else k_q4_rows<bf16_t, 64><<<grid, dim3(64), 0, s>>>(G, (const bf16_t *)q, layer, pos, lens, A, kv_len, (bf16_t *)out);
    }
    return hipGetLastError();
}
