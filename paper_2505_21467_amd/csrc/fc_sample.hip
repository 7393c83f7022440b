// A token and its confidence for every row of logits: temperature, top-k, top-p, min-p, from given uniform numbers.
//
// The entries of a row stand in one order, the larger logit first and the smaller index among equals.  Every filter keeps a prefix of
// that order, and the token is the first entry at which the running sum of the kept weights exceeds u times their total: one
// question asked up to three times, at which entry a running count or sum of the order passes a target.  Nothing is sorted:
//
//  1. k_sample_bins.  Bins of 1/32 of the temperature, on a grid that does not depend on the row: a logit z is in bin floor(32 z / T), its weight
//     over that of the bin's upper edge lies in (0.969, 1] and is held as a whole number of 2^-32.  Each part of a row counts its entries
//     and adds their weights up by bins, 1024 of them down from the part's largest; what is further below weighs less than e^-32.
//  2. k_sample_pick, a workgroup per row.  The parts' bins are added, and running sums over the bins (fp64) say in which bins the targets
//     lie: the entries of those alone, some hundred of 152064, are fetched, from what the parts listed or (by several workgroups where the row is
//     long) from the row, and the targets are found among them by digits of their bits.
//
// Whole sums do not depend on the order in which they are made, so a row gives the same bits whatever else is in the batch and however it is
// cut.  Weights are exact to 2^-32 and their bins' factors to 2^-50 (and to the rounding of 32 z / T, which matters from |z| / T = 2^20 on): with
// sums in fp32, undecided rows would get another token once in a hundred.
#include <math.h>

#include "fc_device.h"
#include "fc_internal.h"
#include "fc_sample.h"

namespace {

constexpr int BINS = 1024, PER_T = 32;       // bins; bins to a unit of z / T
constexpr int SCAN = 512;                    // threads of a part of a row
constexpr int SHORT = 4096, LONG = 16384;    // its entries, at least and at most: their count fits 15 bits, their sum 47
constexpr int PICK = 1024;                   // threads of the second kernel, one to a bin
constexpr int CAP = 12288;                   // entries that it fetches into LDS
constexpr int LISTED = 256, LIST = 1024;     // entries that a part lists, about, and at most
constexpr int FEW = 64;                      // entries that one wave compares with one another
constexpr int ROOM = BINS + 1;               // bins of a part in memory: the one behind its last is 0
constexpr int SUM_BITS = 48;

// exp(-i) and exp(-i / 32): a bin's factor is a product of two.  (The library's function costs 2 us here, most of it for code that is not in the
// instruction cache.)
struct Factors {
    double whole[BINS / PER_T], part[PER_T];
};
constexpr Factors factors()
{
    const double power[5] = {0.36787944117144233, 0.1353352832366127, 0.01831563888873418, 0.00033546262790251185, 1.1253517471925912e-07};  // exp(-2^i)
    Factors f{};
    for (int i = 0; i < BINS / PER_T; ++i) {
        f.whole[i] = 1.;
        for (int k = 0; k < 5; ++k)
            if (i >> k & 1) f.whole[i] *= power[k];
    }
    for (int i = 0; i < PER_T; ++i) {
        double term = 1.;
        for (int k = 1; k < 20; ++k) f.part[i] += term, term *= -(double)i / (PER_T * k);
    }
    return f;
}
static_assert(BINS == 1024 && PER_T == 32, "five powers of 1/e; a wave searches 16 x 64 bins");
__constant__ const Factors FACTORS = factors();

// Order of the entries as a number: the larger logit first, then the smaller index.  -0 is 0.
__device__ __forceinline__ uint64_t rank_of(float z, uint32_t index)
{
    const uint32_t u = __float_as_uint(z + 0.f);
    return (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)~index;
}
__device__ __forceinline__ float logit_of(uint64_t rank)
{
    const uint32_t key = (uint32_t)(rank >> 32);
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// The grid as seen from a largest logit: in which bin below its own a logit is, BINS or more if in none, and its weight over the upper edge's.
struct Grid {
    float most;
    bool infinite;  // then the infinite logits are in bin 0, and no others in any
    double c, by_c, top;  // bins to a unit of logit, 1 / that; the largest logit's bin
    __device__ __forceinline__ Grid(float most_, double c_, double by_c_) : most(most_), infinite(__builtin_amdgcn_readfirstlane(most_ > 3.4028235e38f)), c(c_), by_c(by_c_), top(floor((double)most_ * c_)) {}
    __device__ __forceinline__ int bin(float z, double &within) const
    {
#pragma clang fp contract(off)  // (x is rounded: with one fused operation for x - b an entry's weight would depend on where it is computed)
        const double x = (double)z * c, b = floor(x);
        within = x - b;
        if (infinite) return z == most ? 0 : BINS;
        return (int)fmin(top - b, (double)BINS);  // (NaN: none)
    }
    // exp((within - 1) / 32) in units of 2^-32: with h = 1/64 and |u| <= h, exp(u) by its Taylor series to the fifth power, of which u^5 is given up
    // for what Chebyshev's polynomial says of it, (20 h^2 u^3 - 5 h^4 u) / 16; off by less than 2^-40.
    __device__ __forceinline__ uint64_t weight(double within) const
    {
        if (infinite) return 1ull << 32;
        constexpr double h = 0.5 / PER_T;
        const double u = fma(within, 1.0 / PER_T, -h);
        const double e = fma(u, fma(u, fma(u, fma(u, 1.0 / 24, 1.0 / 6 + h * h / 96), 1.0 / 2), 1.0 - h * h * h * h / 384), 1.0);
        return (uint64_t)__double_as_longlong(fma(e, 0.98449643700540845 * 4294967296.0, 4503599627370496.0)) & 0xfffffffffffffull;  // exp(-h); 2^52 rounds
    }
    // Logits of bins b0 .. b1, and perhaps a few more on either side.
    __device__ __forceinline__ float lowest(int b1) const
    {
        const float x = (float)((top - b1) * by_c);
        return infinite ? most : x - fabsf(x) * 3e-7f;
    }
    __device__ __forceinline__ float highest(int b0) const
    {
        const float x = (float)((top - b0 + 1.) * by_c);
        return infinite ? most : x + fabsf(x) * 3e-7f;
    }
};

// 16 bytes of a row.
template <typename T>
struct Piece {
    static constexpr int N = 16 / sizeof(T), BITS = 8 * sizeof(T);
    T v[N];
    // Entries at .. of a row, -inf from `end` on.  A piece that is not whole is the last 16 bytes shifted (a row of fewer: one by one).
    __device__ __forceinline__ void load(const T *z, int at, int end)
    {
        const int back = min(max(at + N - end, 0), N);
        if (end >= N) *this = __builtin_bit_cast(Piece, fc_load_any<uint4>(z + min(at, end - N)));
        if (back == 0) return;
        if (end < N) {
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = at + j < end ? z[at + j] : fc_from_float<T>(-__builtin_inff());
            return;
        }
        const unsigned __int128 least = (unsigned __int128)LEAST << 64 | LEAST;
        if (back == N) *this = __builtin_bit_cast(Piece, least);
        else *this = __builtin_bit_cast(Piece, __builtin_bit_cast(unsigned __int128, *this) >> (back * BITS) | least << ((N - back) * BITS));
    }
    __device__ __forceinline__ float get(int j) const { return fc_to_float(v[j]); }
    __device__ __forceinline__ void next4()  // the upper half of eight
    {
#pragma unroll
        for (int j = 0; j + 4 < N; ++j) v[j] = v[j + 4];
    }
    static constexpr uint64_t LEAST = sizeof(T) == 2 ? 0xff80ff80ff80ff80ull : 0xff800000ff800000ull;
};

// Every entry of a row's first n: f(index, logit).
template <typename T, int THREADS, typename F>
__device__ __forceinline__ void each_entry(const T *z, int n, F f)
{
    constexpr int N = Piece<T>::N;
#pragma unroll 1
    for (int i0 = threadIdx.x * N; i0 < n; i0 += THREADS * N) {
        Piece<T> x;
        x.load(z, i0, n);
#pragma unroll
        for (int j = 0; j < N; ++j) f(i0 + j, x.get(j));
    }
}

// The value of the lane that CTRL names, 0 where there is none or the row of 16 lanes is not in ROWS.
template <int CTRL, int ROWS, typename X>
__device__ __forceinline__ X from_lane(X x)
{
    struct words { int v[sizeof(X) / 4]; };
    words w = __builtin_bit_cast(words, x);
#pragma unroll
    for (int &v : w.v) v = __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(X, w);
}
// Running results over a wave: one, two, four, eight lanes before within a row of 16, the last lane of the row before, of the half before.
template <typename X, typename F>
__device__ __forceinline__ X wave_run(X x, F f)
{
    x = f(x, from_lane<0x111, 0xf>(x));
    x = f(x, from_lane<0x112, 0xf>(x));
    x = f(x, from_lane<0x114, 0xf>(x));
    x = f(x, from_lane<0x118, 0xf>(x));
    x = f(x, from_lane<0x142, 0xa>(x));
    return f(x, from_lane<0x143, 0xc>(x));
}
template <typename X>
__device__ __forceinline__ X wave_scan(X x)
{
    return wave_run(x, [](X a, X b) { return a + b; });
}

// Sum over the waves before this one, of what every wave's last lane has left in LDS.  (Reads one by one cost 0.3 us more.)
template <int WAVES, typename X>
__device__ __forceinline__ X sum_before(const X *of_wave)
{
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    struct words { int v[sizeof(X) / 4]; };
    words w = __builtin_bit_cast(words, wave_scan(lane < wave ? of_wave[lane % WAVES] : X(0)));
#pragma unroll
    for (int &v : w.v) v = __builtin_amdgcn_readlane(v, 63);
    return __builtin_bit_cast(X, w);
}

// What is kept of a part besides its bins: the largest logit; the last bin of which the list has every entry (-1: none); their number; the last bin
// that is kept (-1: none).
struct __align__(16) Part {
    float largest;
    int32_t bin;
    uint32_t n;
    int32_t last;
};

// One part of a row: bins[] gets (entries << 48 | sum of weights), list[] the ranks of some 256 of its largest entries.
//
// The largest entries of the threads' pieces say where to end: at least as many entries as pieces reach a bin, so with a top-k nothing below the
// bin that k pieces reach can be kept, and is not weighed; the list ends at the bin that 256 reach, or twice
// this part's share of the top-k.
template <typename T, int PART>
__global__ __launch_bounds__(SCAN) void k_sample_bins(FcSampleArgs p, int parts, uint64_t *__restrict__ bins, uint64_t *__restrict__ list,
                                                      Part *__restrict__ about, unsigned long long *__restrict__ shared)
{
    constexpr int N = Piece<T>::N, PIECES = PART / (SCAN * N);
    __shared__ unsigned long long s_bin[BINS];
    __shared__ uint32_t s_count[BINS], s_wave[SCAN / 64], s_n, s_pieces[2];
    __shared__ float s_max[SCAN / 64];
    __shared__ int s_last[2];
    __shared__ uint16_t s_piece[PIECES * SCAN];
    const int tid = threadIdx.x;
    const uint32_t row = blockIdx.x / (uint32_t)parts, part = blockIdx.x - row * parts;
    const int from = part * PART, to = min(p.V, from + PART);
    const T *z = (const T *)p.logits + (size_t)row * p.ld;
    const size_t at = (size_t)row * parts + part;
    Piece<T> x[PIECES];
    float best[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) x[i].load(z, from + (i * SCAN + tid) * N, to);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        best[i] = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < N; ++j) best[i] = fmaxf(best[i], x[i].get(j));  // (NaN is passed over)
    }
    float top = best[0];
#pragma unroll
    for (int i = 1; i < PIECES; ++i) top = fmaxf(top, best[i]);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (tid % 64 == 0) s_max[tid / 64] = top;
    for (int i = tid; i < BINS; i += SCAN) {
        s_bin[i] = 0;
        s_count[i] = 0;
    }
    if (tid == 0) {
        s_last[0] = s_last[1] = BINS;
        s_n = s_pieces[0] = s_pieces[1] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SCAN / 64; ++i) top = fmaxf(top, s_max[i]);
    int end = -1, last = -1;
    if (top > -__builtin_inff()) {
        const Grid g(top, p.inv_t * PER_T, p.bin_width);
        // (in fp32: at most two bins above the exact one)
        const float c = (float)g.c;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const float d = g.infinite ? (best[i] == top ? 0.f : (float)BINS) : (top - best[i]) * c;
            if (d < (float)BINS) atomicAdd(&s_count[(int)d], 1u);
        }
        __syncthreads();
        const uint32_t a = s_count[2 * tid], b = s_count[2 * tid + 1];
        uint32_t run = wave_scan(a + b);
        if (tid % 64 == 63) s_wave[tid / 64] = run;
        __syncthreads();
        run += sum_before<SCAN / 64>(s_wave);
        const uint32_t ks[2] = {p.top_k > 0 ? (uint32_t)p.top_k : 0xffffffffu, (uint32_t)min(max(2 * p.top_k / parts, LISTED), 2 * LISTED)};
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (run >= ks[i] && run - a - b < ks[i]) s_last[i] = run - b >= ks[i] ? 2 * tid : 2 * tid + 1;
        __syncthreads();
        last = min(min(p.last_bin, BINS - 1), s_last[0] + 2);
        end = min(last, s_last[1] + 2);
        const float cut = g.lowest(last);
        // Pieces with an entry that matters are listed, spread over the threads and read again: under a top-k of 50 one entry in hundreds does, and every
        // wave has some.  Those with an entry for the list come first, the others from behind, so that most waves need not ask for places in it.
        const float first_cut = g.lowest(end);
        const bool some_others = __builtin_amdgcn_readfirstlane(end < last);  // (under a small top-k all that matters is listed)
        auto note = [&](uint32_t &number, auto wanted, auto place) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const bool mine = wanted(best[i]);
                const uint64_t in = __ballot(mine);
                if (!in) continue;
                uint32_t base = 0;
                if (tid % 64 == 0) base = atomicAdd(&number, (uint32_t)__builtin_popcountll(in));
                base = __builtin_amdgcn_readfirstlane(base);
                const uint32_t to = __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, base));
                if (mine) s_piece[place(to)] = (uint16_t)(i * SCAN + tid);
            }
        };
        note(s_pieces[0], [&](float x) { return x >= first_cut; }, [](uint32_t to) { return to; });
        if (some_others) note(s_pieces[1], [&](float x) { return x >= cut && !(x >= first_cut); }, [](uint32_t to) { return PIECES * SCAN - 1 - to; });
        __syncthreads();
        const int firsts = (int)s_pieces[0], pieces = firsts + (int)s_pieces[1];
#pragma unroll 1
        for (int i = tid; i < pieces; i += SCAN) {
            const int first = from + s_piece[i < firsts ? i : PIECES * SCAN - 1 - (i - firsts)] * N;
            Piece<T> x;
            x.load(z, first, to);
            // four entries at a time: their chains of fp64 operations overlap, and the wave takes places in the list for all at once
#pragma unroll 1
            for (int j0 = 0; j0 < N; j0 += 4) {
                int bin[4];
                uint64_t w[4], listed[4];
                uint32_t n = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    double within;
                    bin[j] = g.bin(x.get(j), within);
                    w[j] = g.weight(within);
                    listed[j] = __ballot(bin[j] <= end);
                    n += (uint32_t)__builtin_popcountll(listed[j]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (bin[j] <= last) atomicAdd(&s_bin[bin[j]], (unsigned long long)(1ull << SUM_BITS | w[j]));
                if (n && i - tid % 64 < firsts) {
                    const int leader = __builtin_ctzll(__ballot(true));
                    uint32_t place = 0;
                    if (tid % 64 == leader) place = atomicAdd(&s_n, n);
                    place = (uint32_t)__builtin_amdgcn_readlane((int)place, leader);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t own = __builtin_amdgcn_mbcnt_hi((uint32_t)(listed[j] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)listed[j], place));
                        if (bin[j] <= end && own < LIST) list[at * LIST + own] = rank_of(x.get(j), (uint32_t)(first + j0 + j));
                        place += (uint32_t)__builtin_popcountll(listed[j]);
                    }
                }
                x.next4();
            }
        }
    }
    __syncthreads();
    for (int i = tid; i <= last + 1; i += SCAN) bins[at * ROOM + i] = i <= last ? s_bin[i] : 0;
    if (tid == 0 && part == 0) shared[row] = 0;
    if (tid == 0) about[at] = Part{top, s_n <= LIST ? end : -1, min(s_n, (uint32_t)LIST), last};
}

struct Entry {
    uint64_t rank, weight;
};

// Where a row's targets can lie: the bins in which top-k, min-p and top-p end (BINS: none, -1 the end of none) and in which the token is; the last of
// them all; the logits to fetch; whether those are too many for the list; whether no bin in question has more entries than a wave has lanes.
struct Aim {
    int kb, mb, pb0, pb1, sb0, sb1, final, ranges;
    float least[3], most[3];
    bool by_bin, few;
};

struct PickShared {
    double cum[BINS];       // running sums of weights over the bins, from the largest logit down, in units of 2^-32 of bin 0's upper edge
    double factor[BINS];    // exp(-bin / 32)
    uint32_t count[BINS];   // running counts
    uint64_t list[CAP];     // ranks
    uint64_t own[PICK];     // those of one bin, one a thread
    double wave_sum[PICK / 64];
    uint32_t wave_count[PICK / 64];
    uint64_t digit_sum[256];
    uint32_t digit_count[256];
    Entry few[FEW];
    Aim aim;
    unsigned long long ones, zeros, shared, sum_found, rank_found, weight_found;
    uint32_t n, digit, count_found, upto_found;
};

struct Found {
    uint64_t rank, sum, weight;  // the entry, the weight of all up to it, its own
    uint32_t count;              // the number of all up to it
};

// Of n entries, one a lane: number and weight of those before this lane's.
__device__ __forceinline__ uint64_t of_lane(uint64_t x, uint32_t lane)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), (int)lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, (int)lane);
}
__device__ __forceinline__ void before_own(const Entry &own, uint32_t n, uint64_t &weight, uint32_t &count)
{
    for (uint32_t i = 0; i < n; ++i) {
        const uint64_t rank = of_lane(own.rank, i), w = of_lane(own.weight, i);
        weight += rank > own.rank ? w : 0;
        count += rank > own.rank;
    }
}

// Among the n entries that each(f) calls f(rank, weight) for: the one at which the running count or sum, larger ranks first, passes
// `target`; the last one if none does.  Digits of 8 bits from the first bit in which the ranks differ, until a wave can compare what is left.
// ROW: entries come in the order of their index.
template <bool ROW, typename EACH>
__device__ Found select(PickShared &s, bool counting, uint32_t n, uint64_t target, EACH each)
{
    const int tid = threadIdx.x;
    uint64_t low = 0, high = ~0ull, sum = 0;
    uint32_t count = 0;
#pragma unroll 1
    while (n > FEW) {
        __syncthreads();
        if (tid == 0) s.ones = s.zeros = 0;
        if (tid < 256) {
            s.digit_sum[tid] = 0;
            s.digit_count[tid] = 0;
        }
        __syncthreads();
        uint64_t ones = 0, zeros = 0;
        each([&](uint64_t rank, uint64_t) {
            if (rank < low || rank > high) return;
            ones |= rank;
            zeros |= ~rank;
        });
        auto either = [](uint64_t x, uint64_t y) { return x | y; };
        ones = wave_run(ones, either);
        zeros = wave_run(zeros, either);
        if (tid % 64 == 63 && ones) {
            atomicOr(&s.ones, (unsigned long long)ones);
            atomicOr(&s.zeros, (unsigned long long)zeros);
        }
        __syncthreads();
        const int bits = 64 - __builtin_clzll(s.ones & s.zeros), shift = bits > 8 ? bits - 8 : 0;
        const uint32_t mask = (uint32_t)((bits - shift < 8 ? 1u << (bits - shift) : 256u) - 1);
        each([&](uint64_t rank, uint64_t w) {
            if (rank < low || rank > high) return;
            const uint32_t d = (uint32_t)(rank >> shift) & mask;
            uint32_t n = 1;
            if constexpr (ROW) {
                // (equal entries next to one another have one digit and one weight: one addition for all lanes, where 64 to one place took twice the time)
                const uint64_t lanes = __ballot(true);
                const uint32_t d0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)d);
                const uint64_t w0 = of_lane(w, (uint32_t)__builtin_ctzll(lanes));
                if (__ballot(d == d0 && w == w0) == lanes) {
                    if (tid % 64 != __builtin_ctzll(lanes)) return;
                    n = (uint32_t)__builtin_popcountll(lanes);
                }
            }
            atomicAdd((unsigned long long *)&s.digit_sum[d], (unsigned long long)(w * n));
            atomicAdd(&s.digit_count[d], n);
        });
        __syncthreads();
        if (tid < 64) {  // lane i has the digits 255 - 4 i .. 252 - 4 i
            unsigned long long own = 0;
            uint32_t owns = 0;
            for (int i = 0; i < 4; ++i) {
                own += s.digit_sum[255 - 4 * tid - i];
                owns += s.digit_count[255 - 4 * tid - i];
            }
            unsigned long long run = sum + wave_scan(own);
            uint32_t runs = count + wave_scan(owns);
            const uint64_t passed = __ballot(counting ? runs > target : run > target), some = __ballot(owns > 0);
            const int lane = passed ? __builtin_ctzll(passed) : 63 - __builtin_clzll(some);  // (none: the last one with entries)
            if (tid == lane) {
                run -= own;
                runs -= owns;
                int d = 255 - 4 * tid, last = d;
                for (int i = 0; i < 4; ++i, --d) {
                    if (!s.digit_count[d]) continue;
                    last = d;
                    if (counting ? runs + s.digit_count[d] > target : run + s.digit_sum[d] > target) break;
                    run += s.digit_sum[d];
                    runs += s.digit_count[d];
                }
                if (d < 255 - 4 * tid - 3) {  // none passes: the last digit that has entries
                    run -= s.digit_sum[last];
                    runs -= s.digit_count[last];
                }
                s.digit = (uint32_t)last;
                s.sum_found = run;
                s.count_found = runs;
            }
        }
        __syncthreads();
        sum = s.sum_found;
        count = s.count_found;
        n = s.digit_count[s.digit];
        low = (bits < 64 ? s.ones >> bits << bits : 0) | (uint64_t)s.digit << shift;
        high = low | ((1ull << shift) - 1);
    }
    __syncthreads();
    if (tid == 0) s.n = 0;
    __syncthreads();
    each([&](uint64_t rank, uint64_t w) {
        if (rank < low || rank > high) return;
        const uint32_t at = atomicAdd(&s.n, 1u);
        if (at < FEW) s.few[at] = Entry{rank, w};
    });
    __syncthreads();
    n = min(s.n, (uint32_t)FEW);
    if (tid < 64) {
        const Entry own = s.few[tid];
        uint64_t run = sum;
        uint32_t runs = 0;
        before_own(own, n, run, runs);
        const bool passes = counting ? count + runs + 1 > target : run + own.weight > target;
        const bool before = counting ? count + runs > target : run > target;
        if ((uint32_t)tid < n && ((passes && !before) || (!passes && runs == n - 1))) {
            s.rank_found = own.rank;
            s.sum_found = run + own.weight;
            s.weight_found = own.weight;
            s.upto_found = count + runs + 1;
        }
    }
    __syncthreads();
    return Found{s.rank_found, s.sum_found, s.weight_found, s.upto_found};
}

// What select() finds, in one wave without a barrier: entries of bin b in the list, FEW at most.
__device__ __attribute__((noinline)) Found select_few(PickShared &s, bool counting, const Grid g, int listed, int b, uint64_t target)
{
    const int lane = threadIdx.x;
    const float low = g.lowest(b), high = g.highest(b);
    uint32_t n = 0;
#pragma unroll 1
    for (int i = lane; i - lane < listed; i += 64) {
        const uint64_t rank = s.list[min(i, listed - 1)];
        const float x = logit_of(rank);
        double within;
        const bool in = i < listed && x >= low && x <= high && g.bin(x, within) == b;
        const uint64_t mask = __ballot(in);
        const uint32_t to = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, n));
        if (in && to < FEW) s.few[to] = Entry{rank, g.weight(within)};
        n += (uint32_t)__builtin_popcountll(mask);
    }
    n = min(n, (uint32_t)FEW);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const Entry own = s.few[lane];
    uint64_t run = 0;
    uint32_t runs = 0;
    before_own(own, n, run, runs);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const uint64_t to = run + own.weight;
    const bool passes = counting ? runs + 1 > target : to > target, before = counting ? runs > target : run > target;
    const uint64_t mask = __ballot((uint32_t)lane < n && ((passes && !before) || (!passes && runs == n - 1)));
    const int at = mask ? __builtin_ctzll(mask) : 0;
    return Found{(uint64_t)__shfl((unsigned long long)own.rank, at), (uint64_t)__shfl((unsigned long long)to, at), (uint64_t)__shfl((unsigned long long)own.weight, at),
                 (uint32_t)__shfl((int)runs, at) + 1};
}

// The entries of bin b in the list, PICK at most: one a thread.
__device__ __attribute__((noinline)) Found select_one_each(PickShared &s, bool counting, const Grid g, int listed, int b, uint64_t target)
{
    const float low = g.lowest(b), high = g.highest(b);
    double within;
    __syncthreads();
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < listed; i += PICK) {
        const uint64_t rank = s.list[i];
        const float x = logit_of(rank);
        if (!(x >= low && x <= high && g.bin(x, within) == b)) continue;
        const uint32_t at = atomicAdd(&s.n, 1u);
        if (at < PICK) s.own[at] = rank;
    }
    __syncthreads();
    const uint32_t n = min(s.n, (uint32_t)PICK);
    const uint64_t rank = s.own[threadIdx.x];
    g.bin(logit_of(rank), within);
    const uint64_t weight = g.weight(within);
    return select<false>(s, counting, n, target, [&](auto f) {
        if (threadIdx.x < n) f(rank, weight);
    });
}

// The entries of bin b, n of them, in the list or (LIST false) in the row.
template <typename T, bool LIST>
__device__ __attribute__((noinline)) Found select_in(PickShared &s, bool counting, const T *z, int V, const Grid g, int listed, int b, uint32_t n, uint64_t target)
{
    const float low = g.lowest(b), high = g.highest(b);
    return select<!LIST>(s, counting, n, target, [&](auto f) {
        double within;
        if constexpr (LIST) {
#pragma unroll 1
            for (int i = threadIdx.x; i < listed; i += PICK) {
                const uint64_t rank = s.list[i];
                const float x = logit_of(rank);
                if (x >= low && x <= high && g.bin(x, within) == b) f(rank, g.weight(within));
            }
        } else {
            each_entry<T, PICK>(z, V, [&](int i, float x) {
                if (x >= low && x <= high && g.bin(x, within) == b) f(rank_of(x, (uint32_t)i), g.weight(within));
            });
        }
    });
}

// Entries [from, to) of a row with logits in one of n ranges: to the list, as far as there is room.  32 values of a thread are in flight together;
// the few that are wanted are read again.
template <typename T>
__device__ __forceinline__ void fetch(PickShared &s, const T *z, int from, int to, int n, float least0, float most0, float least1, float most1,
                                                float least2, float most2)
{
    constexpr int N = Piece<T>::N, U = 32 / N;
    if (to < N) {  // a row of a few entries
        if ((int)threadIdx.x < to) s.list[atomicAdd(&s.n, 1u)] = rank_of(fc_to_float(z[threadIdx.x]), threadIdx.x);
        return;
    }
#pragma unroll 1
    for (int i0 = from + threadIdx.x * N; i0 < to; i0 += U * PICK * N) {
        Piece<T> x[U];
#pragma unroll
        for (int k = 0; k < U; ++k) x[k] = __builtin_bit_cast(Piece<T>, fc_load_any<uint4>(z + min(i0 + k * PICK * N, to - N)));
        uint32_t left = 0;
#pragma unroll 1
        for (int r = 0; r < n; ++r) {
            const float least = r == 0 ? least0 : r == 1 ? least1 : least2, most = r == 0 ? most0 : r == 1 ? most1 : most2;
#pragma unroll
            for (int k = 0; k < U * N; ++k) left |= x[k / N].get(k % N) >= least && x[k / N].get(k % N) <= most ? 1u << k : 0;
        }
#pragma unroll 1
        while (left) {
            const int k = __builtin_ctz(left), i1 = i0 + k / N * (PICK * N), i = min(i1, to - N) + k % N;
            left &= left - 1;
            if (i < i1) continue;  // (of the last 16 bytes, what another piece has)
            const uint32_t at = atomicAdd(&s.n, 1u);
            if (at < CAP) s.list[at] = rank_of(fc_to_float(z[i]), (uint32_t)i);
        }
    }
}

// Those of one range.  (Apart from the kernel, since it is rare.  What every row runs keeps its registers over the calls in it; only select_in() over
// the row itself saves some in memory.)
template <typename T>
__device__ __attribute__((noinline)) void fetch_range(PickShared &s, const T *z, int V, float least, float most)
{
    fetch(s, z, 0, V, 1, least, most, 0.f, 0.f, 0.f, 0.f);
}

template <typename T>
__global__ __launch_bounds__(PICK) void k_sample_pick(FcSampleArgs p, int parts, const uint64_t *__restrict__ bins, const uint64_t *__restrict__ lists,
                                                      const Part *__restrict__ abouts, unsigned long long *shared, uint64_t *fetched)
{
    __shared__ PickShared s;
    const int tid = threadIdx.x, row = blockIdx.x, slices = gridDim.y, slice = blockIdx.y;
    const T *z = (const T *)p.logits + (size_t)row * p.ld;
    const Part *about = abouts + (size_t)row * parts;
    const uint64_t *part = bins + (size_t)row * parts * ROOM, *lst = lists + (size_t)row * parts * LIST;

    const double factor = FACTORS.whole[tid / PER_T] * FACTORS.part[tid % PER_T];
    float z_max = -__builtin_inff();
    for (int i = tid % 64; i < parts; i += 64) z_max = fmaxf(z_max, about[i].largest);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) z_max = fmaxf(z_max, __shfl_xor(z_max, o));
    if (z_max == -__builtin_inff()) {
        if (tid == 0 && slice == 0) {
            p.tok[row] = -1;
            p.conf[row] = 0.f;
        }
        return;
    }
    const Grid g(z_max, p.inv_t * PER_T, p.bin_width);

    // Thread i: bin i of the row, nine parts in flight together.  (lists_to: the last bin of which the parts' lists have every entry.)
    uint32_t count = 0;
    static_assert(3 * LONG < 1 << (64 - SUM_BITS) && 32 + 16 <= SUM_BITS, "three parts together");
    uint64_t sum = 0;
    uint32_t listed_in = 0;  // (lane: of up to 64 parts)
    int lists_to = BINS;
#pragma unroll 1
    for (int i0 = 0; i0 < parts; i0 += 64) {
        // (lane: part; one of nothing is in no bin)
        double within;
        const int mine = i0 + tid % 64;
        const Part a = about[min(mine, parts - 1)];
        listed_in = a.n;
        const int off = mine < parts ? g.bin(a.largest, within) : BINS;
        lists_to = min(lists_to, off < BINS ? (a.bin < 0 ? -1 : off + a.bin) : BINS);
        const int m = min(parts - i0, 64);
#pragma unroll 1
        for (int i = 0; i < m; i += 9) {
            uint64_t x[9];
#pragma unroll
            for (int k = 0; k < 9; ++k) {
                const int from = min(i + k, m - 1), first = i + k < m ? __builtin_amdgcn_readlane(off, from) : BINS;
                const uint32_t behind = (uint32_t)__builtin_amdgcn_readlane(a.last, from) + 1;
                x[k] = (part + (size_t)(i0 + from) * ROOM)[min((uint32_t)(tid - first), behind)];
            }
#pragma unroll
            for (int k = 0; k < 9; k += 3) {  // (three parts' counts fit 16 bits, and their sums 48)
                const uint64_t y = x[k] + x[k + 1] + x[k + 2];
                count += (uint32_t)(y >> SUM_BITS);
                sum += y & ((1ull << SUM_BITS) - 1);
            }
        }
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) lists_to = min(lists_to, __shfl_xor(lists_to, o));
    double cum = wave_scan((double)sum * factor);
    uint32_t counts = wave_scan(count);
    if (tid % 64 == 63) {
        s.wave_sum[tid / 64] = cum;
        s.wave_count[tid / 64] = counts;
    }
    s.factor[tid] = factor;
    if (tid == 0) s.n = 0;
    __syncthreads();
    cum += sum_before<PICK / 64>(s.wave_sum);
    counts += sum_before<PICK / 64>(s.wave_count);
    s.cum[tid] = cum;
    s.count[tid] = counts;
    __syncthreads();

    auto before = [&](int b) { return b > 0 ? s.cum[b - 1] : 0.; };
    auto counted = [&](int b) { return b > 0 ? s.count[b - 1] : 0u; };
    // The first bin at whose end `enough` holds (it does from there on), BINS if at none: the wave's lanes look at every sixteenth, then at sixteen.
    auto search = [&](auto enough) {
        const int lane = tid % 64;
        const uint64_t sixteen = __ballot(enough(lane * 16 + 15));
        if (!sixteen) return BINS;
        const int b = __builtin_ctzll(sixteen) * 16;
        return b + __builtin_ctzll(__ballot(enough(b + lane % 16)));
    };
    // ... whose running sum reaches x, or (past) exceeds it.
    auto reach = [&](double x, bool past) { return search([&](int b) { return past ? s.cum[b] > x : s.cum[b] >= x; }); };
    const double all = s.cum[BINS - 1], u = p.greedy ? 0. : (double)p.u[row];
    const bool inside = u < 1.;  // (NaN: not)
    // The last bin up to b that has entries (the first has).  Running sums are rounded, by lanes in their own order, so that one may exceed another
    // behind an empty bin.
    auto occupied = [&](int b) {
        const uint32_t n = s.count[b];
        return n > counted(b) ? b : search([&](int b) { return s.count[b] >= n; });
    };
    // The bin of the token for this total of kept weights: where u times it is exceeded.
    auto token_bin = [&](double total) { return occupied(min(reach(fmax(u, 0.) * total, true), BINS - 1)); };

    // Where the targets can lie: the total is known but for the bins in which filters end.  One wave finds out, while the others leave it the compute
    // unit.
    if (tid < 64) {
        double low = all, high = all;
        int kb = BINS, mb = BINS, pb0 = BINS, pb1 = -1;
        if (p.top_k > 0 && s.count[BINS - 1] >= (uint32_t)p.top_k) {  // (otherwise what is kept beyond the bins weighs nothing)
            kb = search([&](int b) { return s.count[b] >= (uint32_t)p.top_k; });
            low = before(kb);
            high = s.cum[kb];
        }
        if (p.top_p < 1.f) {
            pb0 = occupied(min(reach((double)p.top_p * low, false), BINS - 1));
            pb1 = kb < BINS ? occupied(min(reach((double)p.top_p * high, false), BINS - 1)) : pb0;
            low = fmin(low, before(pb0));
            high = fmin(high, s.cum[pb1]);
        }
        if (p.min_p > 0.f && !g.infinite) {
            const double d = g.top - floor((double)z_max * g.c + p.log_min_p * PER_T);
            if (d <= (double)min(kb, BINS - 1)) {  // (beyond the bin in which top-k ends it keeps more)
                mb = (int)d;
                low = fmin(low, before(mb));
                high = fmin(high, s.cum[mb]);
            }
        }
        // (the shortest prefix counts: a filter that ends in a later bin than another one does need not be looked at, but for the top-k whose sum top-p takes)
        if (mb < BINS && pb1 >= 0 && mb > pb1) mb = BINS;
        if (mb < pb0) {
            pb0 = BINS;
            pb1 = -1;
        }
        if (pb1 < 0 && mb < kb) kb = BINS;
        int sb0, sb1;
        if (inside) {
            sb0 = token_bin(low);
            sb1 = low < high ? token_bin(high) : sb0;
        } else {  // the last kept entry: in the first bin in which a filter ends, or, if none of a min-p's bin is kept, in the one before
            sb0 = min(min(kb, mb), pb0);
            sb1 = min(min(kb, mb), pb1 < 0 ? BINS : pb1);
            if (sb1 == BINS) sb0 = sb1 = occupied(BINS - 1);
            else if (sb0 == mb && mb > 0) sb0 = occupied(mb - 1);
        }
        // Logits of the bin in which top-k ends, of those in which the other filters can, and of the token's.  Where they lie apart with many entries
        // between them, three ranges; else one.
        const int f0 = min(pb0, mb), f1 = max(mb < BINS ? mb : -1, pb1), first = min(min(f0, kb), sb0), final = max(max(f1, kb < BINS ? kb : -1), sb1);
        const bool apart = s.count[final] - counted(first) > CAP / 2;
        auto entries = [&](int b0, int b1) { return b0 <= b1 && b1 < BINS ? s.count[b1] - counted(b0) : 0u; };
        if (tid == 0) {
            const float none = __builtin_inff();
            Aim a{kb, mb, pb0, pb1, sb0, sb1, final, 1, {0.f, none, none}, {0.f, -none, -none}, false, false};
            a.least[0] = g.lowest(apart ? sb1 : final);
            a.most[0] = g.highest(apart ? sb0 : first);
            auto add = [&](int b0, int b1) {
                const float least = g.lowest(b1), most = g.highest(b0);
                if (a.ranges == 1) a.least[1] = least, a.most[1] = most;
                else a.least[2] = least, a.most[2] = most;
                ++a.ranges;
            };
            if (apart && f1 >= 0) add(f0, f1);
            if (apart && kb < BINS) add(kb, kb);
            // (too many for the list: bin by bin, then)
            a.by_bin = (apart ? entries(sb0, sb1) + entries(f0, f1) + entries(kb, kb) : entries(first, final)) > (uint32_t)CAP;
            a.few = max(max(entries(kb, kb), entries(mb, mb)), max(entries(pb0, pb1), entries(sb0, sb1))) <= (uint32_t)FEW;
            s.aim = a;
        }
    }
    __syncthreads();
    const Aim aim = s.aim;
    const int kb = aim.kb, mb = aim.mb, pb0 = aim.pb0, pb1 = aim.pb1, sb0 = aim.sb0, sb1 = aim.sb1;
    const bool listed_all = aim.final <= lists_to, by_bin = aim.by_bin && !listed_all;
    auto wanted = [&](float x) {
        bool in = x >= aim.least[0] && x <= aim.most[0];
        if (aim.ranges > 1) in |= (x >= aim.least[1] && x <= aim.most[1]) || (x >= aim.least[2] && x <= aim.most[2]);
        return in;
    };
    if (listed_all) {  // a wave to a part
        if (slice) return;
#pragma unroll 1
        for (int i = __builtin_amdgcn_readfirstlane(tid / 64); i < parts; i += PICK / 64) {
            const uint32_t n = parts <= 64 ? (uint32_t)__builtin_amdgcn_readlane((int)listed_in, i) : about[i].n;
#pragma unroll 1
            for (uint32_t j0 = tid % 64; j0 < n; j0 += 4 * 64) {
                uint64_t r[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) r[k] = lst[(size_t)i * LIST + min(j0 + k * 64, n - 1)];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (j0 + k * 64 < n && wanted(logit_of(r[k]))) {
                        const uint32_t to = atomicAdd(&s.n, 1u);
                        if (to < CAP) s.list[to] = r[k];
                    }
            }
        }
    } else if (by_bin) {
        if (slice) return;
    } else {
        const int per = ((p.V + slices - 1) / slices + 7) / 8 * 8;
        fetch(s, z, slice * per, min(p.V, (slice + 1) * per), aim.ranges, aim.least[0], aim.most[0], aim.least[1], aim.most[1], aim.least[2], aim.most[2]);
        if (slices > 1) {  // the last one to come finds what all have fetched
            __syncthreads();
            const uint32_t own = s.n;
            if (tid == 0) s.shared = atomicAdd(&shared[row], (unsigned long long)own);
            __syncthreads();
            // (Agent-scope stores and loads go past the dies' caches, and a ticket is drawn when the stores have arrived: a fence would write
            // back a whole cache, which took 60 us.)
            uint64_t *of_all = fetched + (size_t)row * CAP;
            const uint32_t at = (uint32_t)s.shared;
            for (uint32_t i = tid; i < own && at + i < (uint32_t)CAP; i += PICK)
                __hip_atomic_store(&of_all[at + i], s.list[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (tid == 0) s.shared = atomicAdd(&shared[row], 1ull << 32);
            __syncthreads();
            if ((uint32_t)(s.shared >> 32) + 1 != (uint32_t)slices) return;
            if (tid == 0) s.n = (uint32_t)s.shared;
            __syncthreads();
            for (uint32_t i = tid; i < min(s.n, (uint32_t)CAP); i += PICK)
                s.list[i] = __hip_atomic_load(&of_all[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    __syncthreads();
    const bool list = s.n <= (uint32_t)CAP && !by_bin;
    const int listed = min((int)s.n, CAP);
    // Where no bin in question has more entries than a wave has lanes, its first wave goes on alone.
    const bool alone = list && listed <= 512 && aim.few;
    if (alone && tid >= 64) return;
    auto sync = [&] {
        if (alone) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        else __syncthreads();
    };
    auto pick = [&](bool counting, int b, uint64_t target) {
        if (alone) return select_few(s, counting, g, listed, b, target);
        const uint32_t n = s.count[b] - counted(b);
        if (list) return n <= PICK ? select_one_each(s, counting, g, listed, b, target) : select_in<T, true>(s, counting, z, p.V, g, listed, b, n, target);
        if (n > (uint32_t)CAP) return select_in<T, false>(s, counting, z, p.V, g, 0, b, n, target);
        __syncthreads();
        if (tid == 0) s.n = 0;
        __syncthreads();
        fetch_range(s, z, p.V, g.lowest(b), g.highest(b));
        __syncthreads();
        const uint32_t all_in = s.n;
        return all_in <= (uint32_t)CAP ? select_in<T, true>(s, counting, z, p.V, g, (int)all_in, b, n, target)
                                       : select_in<T, false>(s, counting, z, p.V, g, 0, b, n, target);
    };

    double total = all;
    uint32_t kept_entries = s.count[BINS - 1];
    if (kb < BINS) {
        kept_entries = (uint32_t)p.top_k;
        const Found f = pick(true, kb, (uint64_t)p.top_k - counted(kb) - 1);
        total = before(kb) + s.factor[kb] * (double)f.sum;
    }
    if (pb1 >= 0) {
        const double x = (double)p.top_p * total;
        const int b = min(max(occupied(min(reach(x, false), BINS - 1)), pb0), pb1);
        const double y = ceil((x - before(b)) / s.factor[b]) - 1.;  // a sum that reaches x passes the whole number below it
        const Found f = pick(false, b, (uint64_t)fmax(y, 0.));
        total = fmin(total, before(b) + s.factor[b] * (double)f.sum);
        kept_entries = min(kept_entries, counted(b) + f.count);
    }
    if (mb < BINS) {  // the last entry that is large enough
        uint64_t kept = 0;
        uint32_t n = 0;
        const float mlow = g.lowest(mb), mhigh = g.highest(mb);
        auto look = [&](float x) {
            double within;
            if (x >= mlow && x <= mhigh && g.bin(x, within) == mb && ((double)x - (double)z_max) * p.inv_t >= p.log_min_p) {
                kept += g.weight(within);
                ++n;
            }
        };
        if (list) {
#pragma unroll 1
            for (int i = tid; i < listed; i += alone ? 64 : PICK) look(logit_of(s.list[i]));
        } else {
            each_entry<T, PICK>(z, p.V, [&](int, float x) { look(x); });
        }
        sync();
        if (tid == 0) {
            s.sum_found = 0;
            s.upto_found = 0;
        }
        sync();
        if (n) {
            atomicAdd(&s.sum_found, (unsigned long long)kept);
            atomicAdd(&s.upto_found, n);
        }
        sync();
        total = fmin(total, before(mb) + s.factor[mb] * (double)s.sum_found);
        kept_entries = min(kept_entries, counted(mb) + s.upto_found);
    }
    // (The last kept entry is found by its number: beside the sum its weight may be nothing.)
    const int b = min(max(inside ? token_bin(total) : search([&](int b) { return s.count[b] >= kept_entries; }), sb0), sb1);
    const double x = (fmax(u, 0.) * total - before(b)) / s.factor[b];
    const Found f = pick(!inside, b, inside ? (uint64_t)fmax(x, 0.) : kept_entries - counted(b) - 1);
    if (tid == 0) {
        p.tok[row] = (int32_t)~(uint32_t)f.rank;
        p.conf[row] = (float)((double)f.weight * s.factor[b] / total);
    }
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// How a call is cut.  Measured over 220 shapes (5001 .. 262144 entries, 1 .. 256 rows, both types) with a top-k of 50 and without one, and over 208 with
// every number of workgroups to a row:
//  - Parts of 4096 where a row has at most 12 of them, 8192 where at most 24, else 16384, and longer where the call has 384 workgroups of the
//    next length: 0.9 % slower than the best length in the mean, 12 at most.  The borders are flat, since short parts are for undecided
//    rows, long ones for a top-k.  bf16, with a top-k and without: one row of 32000 15.7 and 27.3 us by 4096, 16.2 and 29.3 by 8192; 32 x
//    80000 20.4 and 41.9 by 4096, 18.5 and 40.4 by 8192; 32 x 152064 21.0 and 57.4 by 8192, 19.7 and 58.1 by 16384.
//  - Where a row's lists do not do, a workgroup fetches 32768 entries of it at a time.  Rows of 40000 and more have a workgroup for every 20000, as far
//    as there are compute units: 0.6 % slower than the best number in the mean, 5 at most.  bf16 without a top-k: 32 x 152064 57.3 us with
//    one, 48.8 with six, 32 x 80000 40.4 and (four) 37.3, 32 x 40000 34.9 and (two) 33.6, 32 x 36000 30.6 and 32.7.  Workgroups that are not needed cost
//    up to 0.3.
// The workspace has the parts' bins, their lists, what is said about them, and what the slices fetch.
struct Plan {
    int part, parts, slices;
    size_t lists, abouts, shared, fetched, total;
    Plan(int M, int V)
    {
        constexpr int CUS = 256, SLICE = 20000;
        auto parts_of = [&](int entries) { return (V + entries - 1) / entries; };
        part = SHORT;
        while (part < LONG && (parts_of(part) > (part == SHORT ? 12 : 24) || (int64_t)M * parts_of(2 * part) >= 384)) part *= 2;
        parts = parts_of(part);
        slices = M >= CUS ? 1 : CUS / M;
        const int most = V < 2 * SLICE ? 1 : V / SLICE;
        if (slices > most) slices = most;
        const size_t n = (size_t)M * parts;
        lists = align256(n * ROOM * sizeof(uint64_t));
        abouts = lists + align256(n * LIST * sizeof(uint64_t));
        shared = abouts + align256(n * sizeof(Part));
        fetched = shared + align256((size_t)M * sizeof(uint64_t));
        total = fetched + (slices > 1 ? (size_t)M * CAP * sizeof(uint64_t) : 0);
    }
};

template <typename T>
void launch(const FcSampleArgs &p, hipStream_t s)
{
    const Plan w(p.M, p.V);
    char *at = (char *)p.workspace;
    uint64_t *bins = (uint64_t *)at, *lists = (uint64_t *)(at + w.lists), *fetched = (uint64_t *)(at + w.fetched);
    Part *abouts = (Part *)(at + w.abouts);
    unsigned long long *shared = (unsigned long long *)(at + w.shared);
    const dim3 grid((unsigned)(w.parts * p.M));
    if (w.part == LONG) k_sample_bins<T, LONG><<<grid, dim3(SCAN), 0, s>>>(p, w.parts, bins, lists, abouts, shared);
    else if (w.part == 2 * SHORT) k_sample_bins<T, 2 * SHORT><<<grid, dim3(SCAN), 0, s>>>(p, w.parts, bins, lists, abouts, shared);
    else k_sample_bins<T, SHORT><<<grid, dim3(SCAN), 0, s>>>(p, w.parts, bins, lists, abouts, shared);
    k_sample_pick<T><<<dim3((unsigned)p.M, (unsigned)w.slices), dim3(PICK), 0, s>>>(p, w.parts, bins, lists, abouts, shared, fetched);
}

}  // namespace

size_t fc_sample_workspace(int M, int V) { return Plan(M, V).total; }

hipError_t fc_launch_sample(const FcSampleArgs &args, int dtype, hipStream_t s)
{
    FcSampleArgs p = args;
    p.log_min_p = p.min_p > 0.f ? log((double)p.min_p) : 0.;
    p.bin_width = 1. / (p.inv_t * PER_T);
    // With nothing but min-p to sum up to, entries below it need not be counted (two bins for the roundings).
    p.last_bin = BINS - 1;
    if (p.min_p > 0.f && !(p.top_p < 1.f) && -p.log_min_p * PER_T < BINS - 3) p.last_bin = (int)(-p.log_min_p * PER_T) + 2;
    if (dtype == FC_F32) launch<float>(p, s);
    else launch<bf16_t>(p, s);
    return hipGetLastError();
}
