// A token and its confidence for every row of logits: temperature, top-k, top-p, min-p, from given uniform numbers.
//
// The entries of a row stand in one order, the larger logit first and the smaller index among equals.  Every filter keeps a prefix of
// that order, and the token is the first entry at which the running sum of the kept weights exceeds u times their total, so
// everything is one question asked three times: at which entry does a running count or sum of the order exceed a target?
//
// Weights exp((z - z_max) / T) are computed in fp64 and summed as whole numbers, 2^weight_bits for the largest: whole sums do not
// depend on the order, so neither do the token and the confidence on how the row is cut, and a sum that decides between two tokens is
// exact to 2^-44 of the largest weight (a vocabulary of 152064; fp32 sums would pick another token once in a hundred undecided rows).
#include "fc_device.h"
#include "fc_internal.h"
#include "fc_sample.h"

namespace {

constexpr int THREADS = 1024;

// Order-preserving image of a logit; 0: not a number, never chosen.  -0 is 0.
__device__ __forceinline__ uint32_t key_of(float z)
{
    const uint32_t u = __float_as_uint(z + 0.f);
    if (z != z) return 0;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

struct Row {
    float z_max;
    double inv_t, one;  // 1 / T, 2^weight_bits
    __device__ double exact(float z) const { return z == z_max ? 1.0 : exp(((double)z - (double)z_max) * inv_t); }
    __device__ uint64_t weight(float z) const { return (uint64_t)rint(exact(z) * one); }
};

__device__ uint64_t block_sum(uint64_t x, uint64_t *s)
{
    __syncthreads();
    if (threadIdx.x == 0) *s = 0;
    __syncthreads();
    for (int o = 1; o < 64; o <<= 1) x += (uint64_t)__shfl_xor((unsigned long long)x, o);
    if (threadIdx.x % 64 == 0) atomicAdd((unsigned long long *)s, (unsigned long long)x);
    __syncthreads();
    return *s;
}

struct Found {
    uint32_t key;
    uint64_t before;  // count or sum of the entries with larger keys
};

// The key of the entry at which the running sum (count, if !SUM) of the order exceeds `target`, by digits of 8 bits.
template <bool SUM, typename T>
__device__ Found descend(const T *z, int V, const Row &row, uint64_t target, uint64_t *s_bin, uint64_t *s_out)
{
    Found f{0, 0};
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        if (threadIdx.x < 256) s_bin[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < V; i += THREADS) {
            const float x = fc_to_float(z[i]);
            const uint32_t key = key_of(x);
            if (key == 0 || (shift < 24 && (key ^ f.key) >> (shift + 8))) continue;
            const uint64_t w = SUM ? row.weight(x) : 1;
            if (w) atomicAdd((unsigned long long *)&s_bin[key >> shift & 255], (unsigned long long)w);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            uint64_t run = f.before;
            int d = 255;
            for (; d > 0 && run + s_bin[d] <= target; --d) run += s_bin[d];
            s_out[0] = run;
            s_out[1] = (uint64_t)d;
        }
        __syncthreads();
        f.before = s_out[0];
        f.key |= (uint32_t)s_out[1] << shift;
    }
    return f;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void k_sample_rows(FcSampleArgs p)
{
    __shared__ uint64_t s_bin[256], s_out[2], s_sum;
    __shared__ uint32_t s_max;
    __shared__ int s_scan[THREADS];
    const T *z = (const T *)p.logits + (size_t)blockIdx.x * p.ld;
    if (threadIdx.x == 0) s_max = 0;
    __syncthreads();
    uint32_t m = 0;
    for (int i = threadIdx.x; i < p.V; i += THREADS) m = max(m, key_of(fc_to_float(z[i])));
    atomicMax(&s_max, m);
    __syncthreads();
    Row row;
    row.z_max = s_max ? logit_of(s_max) : -__builtin_inff();
    row.inv_t = p.inv_t;
    row.one = p.one;
    if (row.z_max == -__builtin_inff()) {
        if (threadIdx.x == 0) {
            p.tok[blockIdx.x] = -1;
            p.conf[blockIdx.x] = 0.f;
        }
        return;
    }
    uint64_t all = 0, above = 0;
    for (int i = threadIdx.x; i < p.V; i += THREADS) {
        const float x = fc_to_float(z[i]);
        if (x != x) continue;
        const double e = row.exact(x);
        const uint64_t w = (uint64_t)rint(e * row.one);
        all += w;
        if (e >= (double)p.min_p) above += w;
    }
    all = block_sum(all, &s_sum);
    uint64_t total = all;
    if (p.top_k > 0 && p.top_k < p.V) {
        const Found f = descend<false>(z, p.V, row, (uint64_t)p.top_k - 1, s_bin, s_out);
        const uint64_t w = row.weight(logit_of(f.key));
        uint64_t larger = 0;
        for (int i = threadIdx.x; i < p.V; i += THREADS) {
            const float x = fc_to_float(z[i]);
            if (x == x && key_of(x) > f.key) larger += row.weight(x);
        }
        larger = block_sum(larger, &s_sum);
        if (f.key) total = min(total, larger + ((uint64_t)p.top_k - f.before) * w);
    }
    if (p.top_p < 1.f) {
        const uint64_t goal = (uint64_t)ceil((double)p.top_p * (double)total);
        const uint64_t target = goal > 0 ? goal - 1 : 0;
        const Found f = descend<true>(z, p.V, row, target, s_bin, s_out);
        const uint64_t w = row.weight(logit_of(f.key));
        total = min(total, f.before + ((target - f.before) / w + 1) * w);
    }
    if (p.min_p > 0.f) total = min(total, block_sum(above, &s_sum));
    const double u = (double)p.u[blockIdx.x];
    uint64_t target = p.greedy ? 0 : u >= 0. ? (u < 1. ? (uint64_t)(u * (double)total) : total - 1) : u < 0. ? 0 : total - 1;
    target = min(target, total - 1);
    const Found f = descend<true>(z, p.V, row, target, s_bin, s_out);
    const uint64_t w = row.weight(logit_of(f.key));
    const int nth = (int)((target - f.before) / w);  // among the equal ones
    const int chunk = (p.V + THREADS - 1) / THREADS, from = min(p.V, (int)threadIdx.x * chunk), to = min(p.V, from + chunk);
    int n = 0;
    for (int i = from; i < to; ++i) n += key_of(fc_to_float(z[i])) == f.key;
    s_scan[threadIdx.x] = n;
    __syncthreads();
    int before = 0;
    for (int i = 0; i < (int)threadIdx.x; ++i) before += s_scan[i];
    if (before <= nth && nth < before + n) {
        for (int i = from; i < to; ++i)
            if (key_of(fc_to_float(z[i])) == f.key && before++ == nth) p.tok[blockIdx.x] = i;
        p.conf[blockIdx.x] = (float)((double)w / (double)total);
    }
}

}  // namespace

size_t fc_sample_workspace(int dtype, int M, int V) { return 0; }

hipError_t fc_launch_sample(const FcSampleArgs &p, int dtype, hipStream_t s)
{
    if (dtype == FC_F32) k_sample_rows<float><<<dim3((unsigned)p.M), dim3(THREADS), 0, s>>>(p);
    else k_sample_rows<bf16_t><<<dim3((unsigned)p.M), dim3(THREADS), 0, s>>>(p);
    return hipGetLastError();
}
