// A token and its confidence for every row of logits: temperature, top-k, top-p, min-p, from given uniform numbers.
//
// The entries of a row stand in one order, the larger logit first and the smaller index among equals.  Every filter keeps a prefix of
// that order, and the token is the first entry at which the running sum of the kept weights exceeds u times their total: one
// question asked up to three times, at which entry a running count or sum of the order passes a target.  Nothing is sorted:
//
//  1. k_sample_bins.  Bins of 1/32 of the temperature, on a grid that does not depend on the row: a logit z is in bin floor(32 z / T), its weight
//     over that of the bin's upper edge lies in (0.969, 1] and is held as a whole number of 2^-32.  Each part of a row counts its entries
//     and adds their weights up by bins, 1024 of them down from the part's largest; what is further below weighs less than e^-32.
//  2. k_sample_pick, one workgroup per row.  The parts' bins are added, and running sums over the bins (fp64) say in which bins the targets
//     lie: the entries of those alone, some hundred of 152064, are fetched, and the targets are found among them by digits of their bits.
//
// Whole sums do not depend on the order in which they are made, so a row gives the same bits whatever else is in the batch and however it is
// cut.  Weights are exact to 2^-33 and their bins' factors to 2^-53: with sums in fp32, undecided rows would get another token once in a
// hundred.
#include <math.h>

#include "fc_device.h"
#include "fc_internal.h"
#include "fc_sample.h"

namespace {

constexpr int BINS = 1024, PER_T = 32;       // bins; bins to a unit of z / T
constexpr int SCAN = 512, VPT = 32;          // threads and values per thread of a part
constexpr int PART = SCAN * VPT;             // entries of a part: its counts fit 15 bits, its sums 47
constexpr int PICK = 1024;                   // threads of the second kernel, one to a bin
constexpr int CAP = 10240;                   // entries that it fetches into LDS
constexpr uint64_t SUM_BITS = 48;

__host__ __device__ inline int parts_of(int V) { return (V + PART - 1) / PART; }

// Order-preserving image of a logit.  -0 is 0.
__device__ __forceinline__ uint32_t key_of(float z)
{
    const uint32_t u = __float_as_uint(z + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// Bin of a finite logit on the grid, and where it lies in it (0 .. 1 from the lower edge).
struct Place {
    double bin, within;
    __device__ __forceinline__ Place(float z, double c)
    {
        const double x = (double)z * c;
        bin = floor(x);
        within = x - bin;
    }
    // exp((within - 1) / 32) in units of 2^-32: a Taylor series about the middle of the bin, off by less than 2^-45.
    __device__ __forceinline__ uint64_t weight() const
    {
        const double u = (within - 0.5) * (1.0 / PER_T);
        const double e = 1.0 + u * (1.0 + u * (1.0 / 2 + u * (1.0 / 6 + u * (1.0 / 24 + u * (1.0 / 120)))));
        return (uint64_t)__double_as_longlong(e * 0.98449643700540845 * 4294967296.0 + 4503599627370496.0) & 0xfffffffffffffull;  // exp(-1/64); 2^52 rounds
    }
};
// Distance in bins from the one of the largest entry; BINS or more: not in any.  Infinite logits: the largest are in bin 0, at its upper edge.
__device__ __forceinline__ bool in_bins(float z, float z_max, double top, double c, int &bin, uint64_t &w)
{
    if (z == z_max && z > 3.4028235e38f) {
        bin = 0;
        w = 1ull << 32;
        return true;
    }
    const Place p(z, c);
    const double d = top - p.bin;
    if (!(d < (double)BINS)) return false;  // (NaN, and everything below infinity, too)
    bin = (int)d;
    w = p.weight();
    return true;
}

template <typename T>
struct Piece {
    static constexpr int N = 16 / sizeof(T);
    T v[N];
};

// One part of a row: bins[] gets (entries << 48 | sum of weights).
template <typename T>
__global__ __launch_bounds__(SCAN) void k_sample_bins(FcSampleArgs p, int parts, uint64_t *__restrict__ bins, float *__restrict__ largest)
{
    constexpr int N = Piece<T>::N, PIECES = VPT / N;
    __shared__ uint64_t s_bin[BINS];
    __shared__ float s_max[SCAN / 64];
    const int tid = threadIdx.x, part = blockIdx.x, row = blockIdx.y;
    const int from = part * PART, n = min(p.V - from, PART);
    const T *z = (const T *)p.logits + (size_t)row * p.ld + from;
    Piece<T> x[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int at = (i * SCAN + tid) * N;
        if (at + N <= n) x[i] = __builtin_bit_cast(Piece<T>, fc_load_any<uint4>(z + at));
        else
#pragma unroll
            for (int j = 0; j < N; ++j) x[i].v[j] = at + j < n ? z[at + j] : fc_from_float<T>(-__builtin_inff());
    }
#pragma unroll
    for (int i = tid; i < BINS; i += SCAN) s_bin[i] = 0;
    float top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) top = fmaxf(top, fc_to_float(x[i].v[j]));  // (NaN is passed over)
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (tid % 64 == 0) s_max[tid / 64] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SCAN / 64; ++i) top = fmaxf(top, s_max[i]);
    const double c = p.inv_t * PER_T, base = floor((double)top * c);
    if (top > -__builtin_inff()) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                int bin;
                uint64_t w;
                if (in_bins(fc_to_float(x[i].v[j]), top, base, c, bin, w)) atomicAdd((unsigned long long *)&s_bin[bin], (unsigned long long)(1ull << SUM_BITS | w));
            }
    }
    __syncthreads();
    const size_t at = (size_t)row * parts + part;
    for (int i = tid; i < BINS; i += SCAN) bins[at * BINS + i] = s_bin[i];
    if (tid == 0) largest[at] = top;
}

struct PickShared {
    double cum[BINS];       // running sums of weights over the bins, from the largest logit down
    uint32_t count[BINS];   // running counts
    uint64_t sum[BINS];     // the bins' sums, in units of 2^-32 of their upper edge's weight
    uint32_t key[CAP], index[CAP];
    uint16_t bin[CAP];
    uint8_t marked[BINS];
    double wave_sum[PICK / 64];
    uint32_t wave_count[PICK / 64];
    uint64_t digit_sum[256];
    uint32_t digit_count[256];
    uint32_t n, low, high, found[2];
    uint64_t found_sum;
    int first;
};

// Thread i's `x`: the first i for which it holds, BINS if for none.
__device__ int first_bin(PickShared &s, bool x)
{
    __syncthreads();
    if (threadIdx.x == 0) s.first = BINS;
    __syncthreads();
    const uint64_t b = __ballot(x);
    if (b && threadIdx.x % 64 == 0) atomicMin(&s.first, (int)threadIdx.x + __builtin_ctzll(b));
    __syncthreads();
    return s.first;
}

struct Found {
    uint32_t key, count, ties;  // entries with larger keys, and with this one
    uint64_t sum;               // weight of those with larger keys
};

// Among the entries that each(f) calls f(key, weight) for: the key of the one at which the running count (COUNT) or sum, larger keys first, passes
// `target`.  Digits of 8 bits, from the first bit in which the keys differ.
template <bool COUNT, typename EACH>
__device__ Found descend(PickShared &s, uint64_t target, EACH each)
{
    const int tid = threadIdx.x;
    __syncthreads();
    if (tid == 0) {
        s.low = 0xffffffffu;
        s.high = 0;
    }
    __syncthreads();
    uint32_t low = 0xffffffffu, high = 0;
    each([&](uint32_t key, uint64_t) {
        low = min(low, key);
        high = max(high, key);
    });
    for (int o = 1; o < 64; o <<= 1) {
        low = min(low, (uint32_t)__shfl_xor((int)low, o));
        high = max(high, (uint32_t)__shfl_xor((int)high, o));
    }
    if (tid % 64 == 0 && low <= high) {
        atomicMin(&s.low, low);
        atomicMax(&s.high, high);
    }
    __syncthreads();
    int pos = s.low == s.high ? 1 : 32 - __builtin_clz(s.low ^ s.high);  // (one digit of one bit where all are equal)
    Found f{s.high, 0, 0, 0};
    while (pos > 0) {
        const int bits = min(pos, 8), shift = pos - bits;
        __syncthreads();
        if (tid < 256) {
            s.digit_sum[tid] = 0;
            s.digit_count[tid] = 0;
        }
        __syncthreads();
        each([&](uint32_t key, uint64_t w) {
            if (pos < 32 && (key ^ f.key) >> pos) return;
            const uint32_t d = key >> shift & ((1u << bits) - 1);
            atomicAdd((unsigned long long *)&s.digit_sum[d], (unsigned long long)w);
            atomicAdd(&s.digit_count[d], 1u);
        });
        __syncthreads();
        if (tid < 64) {  // lane i has the digits 255 - 4 i .. 252 - 4 i
            uint64_t sum = 0;
            uint32_t count = 0;
            for (int i = 0; i < 4; ++i) {
                sum += s.digit_sum[255 - 4 * tid - i];
                count += s.digit_count[255 - 4 * tid - i];
            }
            uint64_t run = sum;
            uint32_t runs = count;
            for (int o = 1; o < 64; o <<= 1) {
                const uint64_t x = (uint64_t)__shfl_up((unsigned long long)run, o);
                const uint32_t y = (uint32_t)__shfl_up((int)runs, o);
                if (tid >= o) {
                    run += x;
                    runs += y;
                }
            }
            const uint64_t passed = __ballot(COUNT ? f.count + runs > target : f.sum + run > target);
            const int lane = passed ? __builtin_ctzll(passed) : 63;
            if (tid == lane) {
                run += f.sum - sum;
                runs += f.count - count;
                int d = 255 - 4 * tid;
                for (int i = 0; i < 3; ++i, --d) {
                    if (COUNT ? runs + s.digit_count[d] > target : run + s.digit_sum[d] > target) break;
                    run += s.digit_sum[d];
                    runs += s.digit_count[d];
                }
                s.found[0] = (uint32_t)d;
                s.found[1] = runs;
                s.found_sum = run;
            }
        }
        __syncthreads();
        f.key = (pos < 32 ? f.key >> pos << pos : 0) | s.found[0] << shift;
        f.count = s.found[1];
        f.sum = s.found_sum;
        f.ties = s.digit_count[s.found[0]];
        pos = shift;
    }
    return f;
}

template <typename T>
__global__ __launch_bounds__(PICK) void k_sample_pick(FcSampleArgs p, int parts, const uint64_t *__restrict__ bins, const float *__restrict__ largest)
{
    __shared__ PickShared s;
    constexpr int N = Piece<T>::N;
    const int tid = threadIdx.x, row = blockIdx.x;
    const T *z = (const T *)p.logits + (size_t)row * p.ld;
    const double c = p.inv_t * PER_T;

    float z_max = -__builtin_inff();
    for (int i = 0; i < parts; ++i) z_max = fmaxf(z_max, largest[(size_t)row * parts + i]);
    if (z_max == -__builtin_inff()) {
        if (tid == 0) {
            p.tok[row] = -1;
            p.conf[row] = 0.f;
        }
        return;
    }
    const bool infinite = z_max > 3.4028235e38f;
    const double top = floor((double)z_max * c);

    // Thread i: bin i of the row.
    uint32_t count = 0;
    uint64_t sum = 0;
#pragma unroll 4
    for (int i = 0; i < parts; ++i) {
        const float m = largest[(size_t)row * parts + i];
        const double off = infinite ? (m == z_max ? 0. : (double)BINS) : top - floor((double)m * c);  // (a part of nothing is infinitely far)
        const int at = off < (double)BINS ? tid - (int)off : -1;
        const uint64_t x = at >= 0 ? bins[((size_t)row * parts + i) * BINS + at] : 0;
        count += (uint32_t)(x >> SUM_BITS);
        sum += x & ((1ull << SUM_BITS) - 1);
    }
    const double factor = exp(-(double)tid / PER_T);
    double cum = (double)sum * factor;
    uint32_t counts = count;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double x = __shfl_up(cum, o);
        const uint32_t y = (uint32_t)__shfl_up((int)counts, o);
        if (tid % 64 >= o) {
            cum += x;
            counts += y;
        }
    }
    if (tid % 64 == 63) {
        s.wave_sum[tid / 64] = cum;
        s.wave_count[tid / 64] = counts;
    }
    s.sum[tid] = sum;
    s.marked[tid] = 0;
    if (tid == 0) s.n = 0;
    __syncthreads();
    {
        double x = 0.;
        uint32_t y = 0;
        for (int i = 0; i < tid / 64; ++i) {
            x += s.wave_sum[i];
            y += s.wave_count[i];
        }
        cum += x;
        counts += y;
    }
    s.cum[tid] = cum;
    s.count[tid] = counts;
    __syncthreads();
    const double all = s.cum[BINS - 1];
    auto before = [&](int b) { return b > 0 ? s.cum[b - 1] : 0.; };
    auto counted = [&](int b) { return b > 0 ? s.count[b - 1] : 0u; };
    const double u = p.greedy ? 0. : (double)p.u[row];

    // Where the targets can lie: the total is known but for the bins in which filters end.
    double low = all, high = all;
    int kb = BINS, mb = BINS, pb0 = BINS, pb1 = -1;
    if (p.top_k > 0) {
        kb = first_bin(s, counts >= (uint32_t)p.top_k);  // (none: what is kept beyond the bins weighs nothing)
        if (kb < BINS) {
            low = before(kb);
            high = s.cum[kb];
        }
    }
    if (p.top_p < 1.f) {
        pb0 = min(first_bin(s, cum >= (double)p.top_p * low), BINS - 1);
        pb1 = kb < BINS ? min(first_bin(s, cum >= (double)p.top_p * high), BINS - 1) : pb0;
        low = fmin(low, before(pb0));
        high = fmin(high, s.cum[pb1]);
    }
    if (p.min_p > 0.f && !infinite) {
        const double d = top - floor((double)z_max * c + log((double)p.min_p) * PER_T);
        if (d < (double)BINS) {
            mb = (int)d;
            low = fmin(low, before(mb));
            high = fmin(high, s.cum[mb]);
        }
    }
    // The bin in which u times the total lies: the first whose running sum exceeds it, and one with entries.
    auto target_bin = [&](double total) {
        const int b = u < 1. ? first_bin(s, cum > (u > 0. ? u : 0.) * total) : BINS;  // (NaN: none)
        return b < BINS ? b : first_bin(s, cum >= all);
    };
    auto last_bin = [&](double total) { return min(first_bin(s, cum >= total), BINS - 1); };
    const bool inside = u < 1.;
    int sb0 = inside ? target_bin(low) : last_bin(low), sb1 = inside ? (low < high ? target_bin(high) : sb0) : last_bin(high);
    const bool mark = tid == kb || tid == mb || (tid >= pb0 && tid <= pb1) || (tid >= sb0 && tid <= sb1);
    s.marked[tid] = mark;
    if (mark) atomicAdd(&s.n, count);
    __syncthreads();
    const int marked = (int)s.n;
    const bool listed = marked <= CAP;
    __syncthreads();
    if (tid == 0) s.n = 0;
    // No entry below this logit is in a marked bin (a bin to spare for the rounding).
    const int deepest = max(max(sb1, pb1), max(kb < BINS ? kb : 0, mb < BINS ? mb : 0));
    const float lowest = (float)((top - deepest - 1.) / c), cut = infinite ? z_max : lowest - fabsf(lowest) * 1e-6f;
    __syncthreads();

    // Every entry of the row in a bin: f(index, logit, bin, weight).
    auto scan = [&](auto f) {
        for (int i0 = tid * N; i0 < p.V; i0 += PICK * N * 4) {
            Piece<T> x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int at = i0 + k * PICK * N;
                if (at + N <= p.V) x[k] = __builtin_bit_cast(Piece<T>, fc_load_any<uint4>(z + at));
                else
#pragma unroll
                    for (int j = 0; j < N; ++j) x[k].v[j] = at + j < p.V ? z[at + j] : fc_from_float<T>(-__builtin_inff());
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float v = fc_to_float(x[k].v[j]);
                    int bin;
                    uint64_t w;
                    if (v >= cut && in_bins(v, z_max, top, c, bin, w)) f(i0 + k * PICK * N + j, v, bin, w);
                }
        }
    };
    if (listed) {
        scan([&](int i, float v, int bin, uint64_t) {
            if (!s.marked[bin]) return;
            const uint32_t at = atomicAdd(&s.n, 1u);
            s.key[at] = key_of(v);
            s.index[at] = (uint32_t)i;
            s.bin[at] = (uint16_t)bin;
        });
        __syncthreads();
    }
    const int n = listed ? (int)s.n : 0;
    auto weight = [&](float v) {
        int bin;
        uint64_t w = 0;
        in_bins(v, z_max, top, c, bin, w);
        return w;
    };
    // The entries of one bin: f(key, index, weight).
    auto entries = [&](int b, auto f) {
        if (listed) {
            for (int i = tid; i < n; i += PICK)
                if (s.bin[i] == b) f(s.key[i], s.index[i], weight(logit_of(s.key[i])));
        } else {
            scan([&](int i, float v, int bin, uint64_t w) {
                if (bin == b) f(key_of(v), (uint32_t)i, w);
            });
        }
    };
    auto select = [&](auto counting, int b, uint64_t target) {
        return descend<decltype(counting)::value>(s, target, [&](auto f) { entries(b, [&](uint32_t key, uint32_t, uint64_t w) { f(key, w); }); });
    };
    auto scale = [&](int b) { return exp(-(double)b / PER_T); };
    // `x` as a target among the whole numbers of bin b, which has some.
    auto within = [&](int b, double x) {
        const double y = (x - before(b)) / scale(b), most = (double)(s.sum[b] - 1);
        return (uint64_t)(y > 0. ? (y < most ? y : most) : 0.);
    };

    double total = all;
    if (kb < BINS) {
        const uint32_t rest = (uint32_t)p.top_k - counted(kb);  // of this bin, at least one
        const Found f = select(std::true_type(), kb, rest - 1);
        total = before(kb) + scale(kb) * (double)(f.sum + (uint64_t)(rest - f.count) * weight(logit_of(f.key)));
    }
    if (p.top_p < 1.f) {
        const double x = (double)p.top_p * total;
        const int b = min(max(first_bin(s, cum >= x), pb0), pb1);
        const double y = ceil((x - before(b)) / scale(b)) - 1.;  // a sum that reaches x passes the whole number below it
        const uint64_t target = y > 0. ? (y < (double)(s.sum[b] - 1) ? (uint64_t)y : s.sum[b] - 1) : 0;
        const Found f = select(std::false_type(), b, target);
        const uint64_t w = max(weight(logit_of(f.key)), (uint64_t)1);
        total = fmin(total, before(b) + scale(b) * (double)(f.sum + ((target - f.sum) / w + 1) * w));
    }
    if (mb < BINS) {
        uint64_t kept = 0;
        entries(mb, [&](uint32_t key, uint32_t, uint64_t w) {
            if (exp(((double)logit_of(key) - (double)z_max) * p.inv_t) >= (double)p.min_p) kept += w;
        });
        for (int o = 1; o < 64; o <<= 1) kept += (uint64_t)__shfl_xor((unsigned long long)kept, o);
        __syncthreads();
        if (tid == 0) s.found_sum = 0;
        __syncthreads();
        if (tid % 64 == 0) atomicAdd((unsigned long long *)&s.found_sum, (unsigned long long)kept);
        __syncthreads();
        total = fmin(total, before(mb) + scale(mb) * (double)s.found_sum);
        __syncthreads();
    }
    int b;
    uint64_t target;
    if (inside) {
        b = min(max(target_bin(total), sb0), sb1);
        target = within(b, (u > 0. ? u : 0.) * total);
    } else {  // the last kept entry
        b = min(max(last_bin(total), sb0), sb1);
        const double y = rint((total - before(b)) / scale(b)) - 1.;
        target = y > 0. ? (y < (double)(s.sum[b] - 1) ? (uint64_t)y : s.sum[b] - 1) : 0;
    }
    const Found f = select(std::false_type(), b, target);
    const uint64_t w = max(weight(logit_of(f.key)), (uint64_t)1), nth = min((target - f.sum) / w, (uint64_t)f.ties - 1);
    // Among equal ones by the index, smaller ones first.
    const Found g = descend<true>(s, nth, [&](auto f2) {
        entries(b, [&](uint32_t key, uint32_t index, uint64_t) {
            if (key == f.key) f2(~index, 0);
        });
    });
    if (tid == 0) {
        p.tok[row] = (int32_t)~g.key;
        p.conf[row] = (float)((double)w * scale(b) / total);
    }
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

size_t fc_sample_workspace(int dtype, int M, int V)
{
    const size_t parts = (size_t)M * parts_of(V);
    return align256(parts * BINS * sizeof(uint64_t)) + parts * sizeof(float);
}

hipError_t fc_launch_sample(const FcSampleArgs &p, int dtype, hipStream_t s)
{
    const int parts = parts_of(p.V);
    uint64_t *bins = (uint64_t *)p.workspace;
    float *largest = (float *)((char *)p.workspace + align256((size_t)p.M * parts * BINS * sizeof(uint64_t)));
    const dim3 grid((unsigned)parts, (unsigned)p.M);
    if (dtype == FC_F32) {
        k_sample_bins<float><<<grid, dim3(SCAN), 0, s>>>(p, parts, bins, largest);
        k_sample_pick<float><<<dim3((unsigned)p.M), dim3(PICK), 0, s>>>(p, parts, bins, largest);
    } else {
        k_sample_bins<bf16_t><<<grid, dim3(SCAN), 0, s>>>(p, parts, bins, largest);
        k_sample_pick<bf16_t><<<dim3((unsigned)p.M), dim3(PICK), 0, s>>>(p, parts, bins, largest);
    }
    return hipGetLastError();
}
