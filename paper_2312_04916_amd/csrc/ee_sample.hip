// Choosing tokens (ee_sample of ee.h): one kernel passes over the logits and leaves a few numbers of each run of tokens, a second one
// finds a row's token from them and from the few runs that matter, a third one does so for rows in which too many tokens may be kept.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ee_exp.h"
#include "ee_lanes.h"
#include "ee_launch.h"
#include "ee_sample.h"

namespace ee {

namespace {

typedef unsigned long long u64;

constexpr int ONE = 44;  // weights are multiples of 2^-44 of the largest: 2^18 of them stay below 2^62
constexpr int CHUNKS = SAMPLE_RUN / SAMPLE_CHUNK, RUNS = (1 << 18) / SAMPLE_RUN;
constexpr int LIST = 256;  // elements of a bin that are ranked one by one
constexpr float MOST_FLOAT = 3.4028235e38f;

// Order of the floats as unsigned numbers; -0 counts as 0, NaN as the largest.
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);
    return z != z ? 0xffffffffu : b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
constexpr uint32_t KEY_INF = 0xff800000u, KEY_NINF = 0x007fffffu;

// 2^y * 2^shift for y <= 0.  In 64 bits: the place of u * total among the sums has to be found in runs of 2^18 weights.  2^f on
// [-1/2, 1/2] is a polynomial through nine Chebyshev nodes, its constant term kept at 1 (error 2^-45); adding 1.5 * 2^52 leaves the
// nearest whole number in the low bits, and exponents are added as they are (rounding, conversion and scaling instructions for 64 bits
// take four times as long as additions).
__device__ __forceinline__ double power_of(double y, int shift) {
    const double t = fmax(y, -900.0) + 0x1.8p52, f = fmax(y, -900.0) - (t - 0x1.8p52);
    double g = 0x1.b63880a30e9ffp-24;
    g = fma(g, f, 0x1.63d136366db24p-20);
    g = fma(g, f, 0x1.ffcb9515a8016p-17);
    g = fma(g, f, 0x1.4308ac85aa947p-13);
    g = fma(g, f, 0x1.5d87fe86fe88ep-10);
    g = fma(g, f, 0x1.3b2ab7181b755p-7);
    g = fma(g, f, 0x1.c6b08d7047e52p-5);
    g = fma(g, f, 0x1.ebfbdff823cedp-3);
    g = fma(g, f, 0x1.62e42fefa39efp-1);
    const u64 m = (u64)__double_as_longlong(fma(g, f, 1.0));
    const uint32_t n = (uint32_t)__double_as_longlong(t) + (uint32_t)shift;
    return __longlong_as_double((long long)((u64)((uint32_t)(m >> 32) + (n << 20)) << 32 | (uint32_t)m));
}
// exp((z - top) / temperature) as a whole number of 2^-44, with per_t = log2(e) / temperature; adding 2^52 rounds to one and leaves it in the
// low bits.
__device__ __forceinline__ u64 weight_of(float z, float top, double per_t) {
    return (u64)__double_as_longlong(power_of(((double)z - (double)top) * per_t, ONE) + 0x1p52) & ((1ull << 52) - 1);
}
// The same with the bits of 2^52 on top: sums of n of them are the weights' sum and n times that, modulo 2^64.
__device__ __forceinline__ u64 weight_bits(float z, float top, double per_t) {
    return (u64)__double_as_longlong(power_of(((double)z - (double)top) * per_t, ONE) + 0x1p52);
}
constexpr u64 BITS = 0x4330000000000000ull;
// a sum of weights relative to one top as one relative to another, 2^-y times as large
__device__ __forceinline__ u64 rescaled(u64 sum, double y) { return y == 0 ? sum : (u64)rint((double)sum * power_of(y, 0)); }

// A value of the lane 1, 2, 4, 8 before in the row of 16 (0x110 + n), of the last lane of the row before (0x142, to rows 1 and 3), of the
// first half (0x143, to rows 2 and 3); 0 where there is none.
template <int FROM, int ROWS = 0xf>
__device__ __forceinline__ uint32_t lanes_before(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, FROM, ROWS, 0xf, false);
}
template <int FROM, int ROWS = 0xf>
__device__ __forceinline__ u64 lanes_before(u64 v) {
    return (u64)lanes_before<FROM, ROWS>((uint32_t)(v >> 32)) << 32 | lanes_before<FROM, ROWS>((uint32_t)v);
}
// inclusive sums of the first N lanes, in their order
template <int N = 64, typename T>
__device__ __forceinline__ T wave_scan(T v) {
    v += lanes_before<0x111>(v);
    v += lanes_before<0x112>(v);
    v += lanes_before<0x114>(v);
    if constexpr (N > 8) v += lanes_before<0x118>(v);
    if constexpr (N > 16) {
        v += lanes_before<0x142, 0xa>(v);
        v += lanes_before<0x143, 0xc>(v);
    }
    return v;
}
__device__ __forceinline__ uint32_t last_lane(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, 63); }
__device__ __forceinline__ u64 last_lane(u64 v) { return (u64)last_lane((uint32_t)(v >> 32)) << 32 | last_lane((uint32_t)v); }
template <typename T>
__device__ __forceinline__ T wave_total(T v) {
    return last_lane(wave_scan(v));
}
__device__ __forceinline__ double wave_total(double v) {  // (in an order of its own: the same every time)
    for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
    return v;
}
// largest of a wave's numbers
__device__ __forceinline__ uint32_t wave_most(uint32_t v) {
    v = max(v, lanes_before<0x111>(v));
    v = max(v, lanes_before<0x112>(v));
    v = max(v, lanes_before<0x114>(v));
    v = max(v, lanes_before<0x118>(v));
    v = max(v, lanes_before<0x142, 0xa>(v));
    v = max(v, lanes_before<0x143, 0xc>(v));
    return last_lane(v);
}

// f * sum for 0 <= f < 1, rounded down (up): 24 bits of f times 62 of the sum, exactly.
__device__ __forceinline__ u64 share_of(float f, u64 sum, bool up) {
    const uint32_t b = __float_as_uint(f) & 0x7fffffffu, e = b >> 23;  // (-0 is 0)
    const u64 mantissa = e ? (b & 0x7fffff) | 0x800000 : b;
    const int s = 150 - (int)max(e, 1u);  // f = mantissa / 2^s, 24 <= s < 150
    const u64 lo = sum * mantissa, hi = __umul64hi(sum, mantissa);  // below 2^86
    if (s >= 86) return up && mantissa && sum;
    const u64 q = s < 64 ? hi << (64 - s) | lo >> s : hi >> (s - 64);
    const u64 rest = s < 64 ? lo << (64 - s) : lo | (s > 64 ? hi << (128 - s) : 0);
    return q + (up && rest);
}

struct Settings {
    float u, t, top_p, min_p;
    int top_k;
    bool bad, greedy, by_k, by_p, by_m;
    double per_t;
    __device__ __forceinline__ Settings(const Sampling& p, int r) {
        u = p.u[r], t = p.temperature ? p.temperature[r] : p.one_temperature;
        top_k = p.top_k ? p.top_k[r] : p.one_top_k;
        top_p = p.top_p ? p.top_p[r] : p.one_top_p, min_p = p.min_p ? p.min_p[r] : p.one_min_p;
        bad = !(u >= 0.f && u < 1.f) || !(t >= 0.f && t < INFINITY) || top_k < 0 || !(top_p >= 0.f && top_p <= 1.f) || !(min_p >= 0.f && min_p <= 1.f);
        greedy = t == 0.f;
        by_k = !greedy && top_k > 0 && top_k < p.vocab, by_p = !greedy && top_p < 1.f, by_m = !greedy && min_p > 0.f;
        per_t = greedy || bad ? 0.0 : 1.4426950408889634 / (double)t;
    }
    // whether the sum of all weights matters: with top-k or min-p alone what is kept is summed up when it is known
    __device__ __forceinline__ bool whole_sum() const { return !bad && !greedy && !by_k && (by_p || !by_m); }
};

// Four neighbouring elements, -inf behind the row's end.  (Each lane branches between one load and four: the compiler puts a wait for all loads
// before the next one of the other arm, so that a wave has one of these on its way, however many are asked for ahead.  Rows that
// are not aligned are read element by element: 512 rows of 50 257 logits in bf16, temperature alone, take 56 us for 41.)
template <typename T>
__device__ __forceinline__ void load4(const T* z, int i, int n, bool vec, float (&v)[4]) {
    if (vec && i + 4 <= n) {
        if constexpr (sizeof(T) == 2) {
            const uint2 a = *(const uint2*)(z + i);
            v[0] = __uint_as_float(a.x << 16), v[1] = __uint_as_float(a.x & 0xffff0000u);
            v[2] = __uint_as_float(a.y << 16), v[3] = __uint_as_float(a.y & 0xffff0000u);
        } else {
            const float4 a = *(const float4*)(z + i);
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = i + j < n ? (float)z[i + j] : -INFINITY;
    }
}

// ------------------------------------------------------------------------------------------------
// the pass over the logits: a wave takes `each` runs of 1024 tokens, one after the other.  512 rows of 50 304 logits in fp32 take 40 us
// where all weights are summed up and 22 where they are not (4.7 TB/s): the 64-bit arithmetic (16 instructions a logit, 18 us) adds to the
// time of the loads, which do not run ahead of it (load4).
// ------------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void sample_runs_kernel(Sampling p, int each) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const SampleRow at(p.vocab);
    const uint32_t all = (uint32_t)p.rows * at.runs, i0 = (uint32_t)wave * each, i1 = min(all, i0 + each);
    if (i0 >= i1) return;
    const bool scores = p.logprob || p.confidence;
    int r = i0 / (uint32_t)at.runs, run = i0 - r * at.runs;
    Settings s(p, r);
    float next[4][4];
    auto load = [&](int r, int run) {
        const T* z = (const T*)p.logits + (int64_t)r * p.row_stride;
#pragma unroll
        for (int j = 0; j < 4; ++j) load4(z, run * SAMPLE_RUN + j * 256 + lane * 4, p.vocab, p.vec, next[j]);
    };
    load(r, run);
    for (uint32_t i = i0; i < i1; ++i) {
        float v[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[j][k] = next[j][k];
        const int r_now = r, run_now = run;
        if (++run == at.runs) run = 0, ++r;
        if (i + 1 < i1) load(r, run);
        char* out = p.workspace + (size_t)r_now * at.bytes();
        bool nan = false;
        float top[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            nan |= __builtin_isunordered(v[j][0], v[j][1]) || __builtin_isunordered(v[j][2], v[j][3]);
            float m = fmaxf(fmaxf(v[j][0], v[j][1]), fmaxf(v[j][2], v[j][3]));
            m = fmaxf(m, row_rotate<8>(m)), m = fmaxf(m, row_rotate<4>(m)), m = fmaxf(m, row_rotate<2>(m)), m = fmaxf(m, row_rotate<1>(m));
            top[j] = m;
        }
        const float most = rows4_max(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
        if (__ballot(nan)) top[0] = top[1] = top[2] = top[3] = __uint_as_float(0x7fc00000u);
        if ((lane & 15) == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) ((float*)out)[run_now * CHUNKS + j * 4 + (lane >> 4)] = top[j];
        }
        const float ref = fmaxf(most, -MOST_FLOAT);
        if (s.whole_sum()) {
            u64 sum = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) sum += weight_bits(v[j][k], ref, s.per_t);
            sum = wave_scan(sum - 16 * BITS);
            if (lane == 63) ((u64*)(out + at.sums()))[run_now] = sum;
        }
        if (scores) {
            float part[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                part[j] = (exp_of(v[j][0] - ref) + exp_of(v[j][1] - ref)) + (exp_of(v[j][2] - ref) + exp_of(v[j][3] - ref));
            const float raw = wave_sum((part[0] + part[1]) + (part[2] + part[3]));
            if (lane == 0) ((float*)(out + at.raws()))[run_now] = raw;
        }
        if (r != r_now && i + 1 < i1) s = Settings(p, r);
    }
}

// ------------------------------------------------------------------------------------------------
// a row's token
// ------------------------------------------------------------------------------------------------

// What has been found out about a row: kept are the elements above `key` and the first `ties` of the ones that equal it, by index (all of
// them, if not `some`).
struct Cut {
    uint32_t key;
    int ties, some;
    u64 weight;  // of all that is kept
};
__device__ __forceinline__ Cut nothing_cut() { return Cut{0, 1 << 30, 0, 0}; }

// The threads that look for a row's cut: a whole workgroup, or one wave of it, which needs no barriers.
template <int NT>
__device__ __forceinline__ void meet() {
    if constexpr (NT == 64)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (LDS serves a wave in its order)
    else
        __syncthreads();
}

template <int NT, int N_BINS>
struct CutShared {
    u64 sums[NT / 64];
    uint32_t counts[NT / 64];
    u64 bin_weight[N_BINS];
    uint32_t bin_count[N_BINS];
    uint32_t list[LIST], list_index[LIST];  // the elements of the cut's bin, if they are few
    u64 list_weight[LIST];
    uint32_t n_list, lo, hi;  // keys of the bin that is looked into
    int bin, listed;
    u64 base_weight;
    uint32_t base_count, in_bin;
    Cut cut;
};

__device__ __forceinline__ uint32_t of_lane(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ u64 of_lane(u64 v, int lane) { return (u64)of_lane((uint32_t)(v >> 32), lane) << 32 | of_lane((uint32_t)v, lane); }

// Sums over the threads: exclusive prefix of each one's value, and the total.  `waves` is still read here when a thread returns: it may be
// written again behind the next meeting, not before.
template <int NT, typename T>
__device__ __forceinline__ T before_me(T v, T& total, T* waves) {
    const T in = wave_scan(v);
    if constexpr (NT == 64) {
        total = last_lane(in);
        return in - v;
    } else {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (lane == 63) waves[wave] = in;
        __syncthreads();
        const T sums = wave_scan<NT / 64>(lane < NT / 64 ? waves[lane] : (T)0);  // (of the waves, one in a lane)
        total = of_lane(sums, NT / 64 - 1);
        return in - v + (wave ? of_lane(sums, wave - 1) : (T)0);
    }
}

// Bins share the distance to the top, `per_bin` to one.
__device__ __forceinline__ int bin_at(float z, float top, float per_bin, int bins) { return (int)fminf((top - z) * per_bin, (float)(bins - 1)); }

// Counts and weights of the elements into the bins, which are empty.  E: each(f) calls f(key, index, weight()) for a thread's elements, and
// each(lo, hi, f) for those whose logit is in [lo, hi] (and may for others); list() puts the elements of a bin by distance into s.list,
// if it can.
template <int NT, int N_BINS, typename E, typename B>
__device__ __forceinline__ void fill_bins(const E& elements, CutShared<NT, N_BINS>& s, B bin_of) {
    // (what lies furthest may be most of a row: it is counted apart, not at one place by all)
    uint32_t last_count = 0;
    u64 last_weight = 0;
    elements.each([&](uint32_t key, int, auto weight) {
        const int b = bin_of(key);
        if (b < 0) return;
        const u64 w = weight();
        if (b == N_BINS - 1) {
            ++last_count, last_weight += w;
        } else {
            atomicAdd(&s.bin_count[b], 1u);
            atomicAdd(&s.bin_weight[b], w);
        }
    });
    if (last_count) atomicAdd(&s.bin_count[N_BINS - 1], last_count), atomicAdd(&s.bin_weight[N_BINS - 1], last_weight);
    meet<NT>();
}
template <int NT, int N_BINS>
__device__ __forceinline__ void empty_bins(CutShared<NT, N_BINS>& s, int tid) {
#pragma unroll
    for (int i = 0; i < N_BINS / NT; ++i) s.bin_weight[tid + i * NT] = 0, s.bin_count[tid + i * NT] = 0;
}

// The last element that is kept where elements are kept, in their order, as long as fewer than `limit` came before (BY_COUNT) or
// their weights' sum is below `limit`: the bin in which that happens, then its elements one by one, or finer bins if they are many,
// which share the keys that are in the bin, until it holds one key only.  If all are kept, the cut is left as it was.
// The bins by distance are filled; false: they no longer are.
template <bool BY_COUNT, int NT, int N_BINS, typename E>
__device__ bool find_cut(const E& elements, CutShared<NT, N_BINS>& s, u64 limit, float top, float per_bin) {
    constexpr int PER = N_BINS / NT, RANK = NT == 64 ? 64 : LIST;  // (n^2 / NT comparisons: 256 by one wave took 90 us)
    const int tid = threadIdx.x & (NT - 1), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint32_t lo = 0, hi = 0;
    int shift = -1;  // -1: bins by distance
    u64 base_weight = 0;
    uint32_t base_count = 0;
    for (;;) {
        auto bin_of = [&](uint32_t key) {
            if (shift < 0) return bin_at(value_of(key), top, per_bin, N_BINS);
            return key >= lo && key <= hi ? (int)((hi - key) >> shift) : -1;
        };
        // (a thread's bins lie next to one another)
        uint32_t c[PER], c_all = 0;
        u64 w[PER], w_all = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) c[i] = s.bin_count[tid * PER + i], w[i] = s.bin_weight[tid * PER + i], c_all += c[i], w_all += w[i];
        const uint32_t c_in = wave_scan(c_all);
        const u64 w_in = wave_scan(w_all);
        if (lane == 63) s.counts[wave] = c_in, s.sums[wave] = w_in;
        if (tid == 0) s.n_list = 0, s.lo = 0xffffffffu, s.hi = 0, s.bin = -1, s.listed = 0;
        meet<NT>();
        uint32_t c_before = base_count + c_in - c_all;
        u64 w_before = base_weight + w_in - w_all;
        if constexpr (NT > 64) {
            const uint32_t c_waves = wave_scan<NT / 64>(lane < NT / 64 ? s.counts[lane] : 0u);
            const u64 w_waves = wave_scan<NT / 64>(lane < NT / 64 ? s.sums[lane] : 0ull);
            if (wave) c_before += of_lane(c_waves, wave - 1), w_before += of_lane(w_waves, wave - 1);
        }
        // the bin in which the limit is reached
        if (BY_COUNT ? c_before < limit && c_before + c_all >= limit : w_before < limit && w_before + w_all >= limit) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (c[i] && (BY_COUNT ? c_before < limit && c_before + c[i] >= limit : w_before < limit && w_before + w[i] >= limit))
                    s.bin = tid * PER + i, s.base_count = c_before, s.base_weight = w_before, s.in_bin = c[i];
                c_before += c[i], w_before += w[i];
            }
        }
        meet<NT>();
        const int bin = s.bin;
        if (bin < 0) {  // all are kept
            meet<NT>();
            return shift < 0;
        }
        base_count = s.base_count, base_weight = s.base_weight;
        const uint32_t in_bin = s.in_bin;
        uint32_t key_lo = 0xffffffffu, key_hi = 0;
        if (!(shift < 0 && in_bin <= RANK && elements.list(s, bin))) {
            // (the bin's logits lie between these, and little else)
            const float far = fabsf(top) * 1e-6f + (float)(bin + 1) / per_bin * 1e-5f;
            // (per_bin is 0 where the spread is infinite: fmaxf and fminf drop what is then no number)
            const float z_lo = shift >= 0 ? value_of(lo) : bin == N_BINS - 1 ? -INFINITY : fmaxf(top - (float)(bin + 1) / per_bin - far, -INFINITY);
            const float z_hi = shift >= 0 ? value_of(hi) : fminf(top - (float)bin / per_bin + far, INFINITY);
            elements.each(z_lo, z_hi, [&](uint32_t key, int index, auto weight) {
                if (bin_of(key) == bin) {
                    key_lo = min(key_lo, key), key_hi = max(key_hi, key);
                    if (in_bin <= RANK) {
                        const uint32_t at = atomicAdd(&s.n_list, 1u);
                        s.list[at] = key, s.list_index[at] = index, s.list_weight[at] = weight();
                    }
                }
            });
        }
        if (in_bin > RANK && key_lo <= key_hi) atomicMin(&s.lo, key_lo), atomicMax(&s.hi, key_hi);
        meet<NT>();
        if (in_bin <= RANK) {
            const int n = (int)s.n_list;
            if (tid == 0) s.listed = shift < 0;  // (whole)
            // so many lanes for each that all threads have work, 16 at most
            int lanes = 1;
            while (lanes < 16 && 2 * lanes * n <= NT) lanes *= 2;
            for (int e0 = 0; e0 < n; e0 += NT / lanes) {
                const int e = e0 + tid / lanes;
                const uint32_t key = e < n ? s.list[e] : 0;
                const u64 each = e < n ? s.list_weight[e] : 0;
                uint32_t above = 0, equal = 0;
                u64 weight = 0;
                for (int i = tid & (lanes - 1); i < n; i += lanes) {
                    const uint32_t k = s.list[i];
                    if (k > key) ++above, weight += s.list_weight[i];
                    if (k == key) ++equal;
                }
                for (int d = 1; d < lanes; d *= 2) {
                    above += __shfl_xor((int)above, d), equal += __shfl_xor((int)equal, d);
                    weight += (u64)__shfl_xor((long long)weight, d);
                }
                above += base_count, weight += base_weight;
                const bool mine = e < n && (BY_COUNT ? above < limit && above + equal >= limit : weight < limit && weight + equal * each >= limit);
                if (mine) {  // (all of one key write the same)
                    const u64 ties = BY_COUNT ? limit - above : (limit - weight + each - 1) / each;
                    s.cut = Cut{key, (int)ties, ties < equal, weight + ties * each};
                }
            }
            meet<NT>();
            return shift < 0;
        }
        lo = s.lo, hi = s.hi;
        if (lo == hi) {  // one key: so many of them
            if (tid == 0) {
                const u64 each = s.bin_weight[bin] / in_bin;
                const u64 ties = BY_COUNT ? limit - base_count : (limit - base_weight + each - 1) / each;
                s.cut = Cut{lo, (int)ties, ties < in_bin, base_weight + ties * each};
            }
            meet<NT>();
            return shift < 0;
        }
        shift = max(0, 32 - __builtin_clz(hi - lo) - (31 - __builtin_clz(N_BINS)));
        empty_bins(s, tid);
        meet<NT>();
        fill_bins(elements, s, bin_of);
    }
}

__device__ __forceinline__ void write_row(const Sampling& p, int r, int token, float z, float top, double raw, double log_raw) {
    p.token[r] = token;
    if (p.logprob) p.logprob[r] = (float)((double)z - (double)top - log_raw);
    if (p.confidence) p.confidence[r] = (float)(1.0 / raw);
}

constexpr int ROW_THREADS = 512, ROW_WAVES = ROW_THREADS / 64;
constexpr int CANDIDATES = 2048;        // that the threads hold
constexpr int WAVE_CANDIDATES = 1024;   // that a wave may find
constexpr int ONE_WAVE = 512;           // candidates that one wave takes
constexpr int AT_ONCE = 16;             // runs of 64 tokens that a wave asks for at once

struct RowShared {
    union {
        CutShared<ROW_THREADS, ROW_THREADS> all;
        CutShared<64, ROW_THREADS> one;
    };
    u64 sums[ROW_WAVES];
    uint32_t tops[ROW_WAVES], lows[ROW_WAVES], founds[ROW_WAVES], places[ROW_WAVES], floors[ROW_WAVES];
    double raw[ROW_WAVES];
    double log_raw;
    uint32_t place, found, candidates;
    uint32_t floor_count[ROW_THREADS];
    int floor_bin;
    u64 left;
    float ref;
    uint16_t chunks[(1 << 18) / SAMPLE_CHUNK];
    float2 found_at[ROW_WAVES][WAVE_CANDIDATES];  // logit, and the bits of the index
};

// Candidates that threads hold.
template <int OWN>
struct OwnElements {
    uint32_t key[OWN], index[OWN];
    u64 weight[OWN];
    int n;
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int j = 0; j < OWN; ++j)
            if (j < n) f(key[j], 0, [&] { return weight[j]; });
    }
    template <typename F>
    __device__ __forceinline__ void each(float, float, F f) const {
        each(f);
    }
    template <typename S>
    __device__ __forceinline__ bool list(S&, int) const {
        return false;
    }
};

// The token among n candidates, which lie in s.found_at in the order of their indices, from[] of them before each wave's; held by NT
// threads, OWN each, neighbouring ones by a thread.
template <int NT, int OWN, typename S>
__device__ void token_of(const Settings& g, RowShared& s, S& c, const uint32_t (&from)[ROW_WAVES], int n, float top, float least_z, double reach, u64 total) {
    const int tid = threadIdx.x & (NT - 1);
    const int mine = (n + NT - 1) / NT, at0 = tid * mine;
    OwnElements<OWN> own;
    own.n = max(0, min(mine, n - at0));
    u64 part = 0;
#pragma unroll
    for (int j = 0; j < OWN; ++j) {
        int w = 0, i = at0 + j;
#pragma unroll
        for (int k = 1; k < ROW_WAVES; ++k)
            if (at0 + j >= (int)from[k]) w = k, i = at0 + j - (int)from[k];
        own.key[j] = 0, own.index[j] = 0, own.weight[j] = 0;
        if (j < own.n) {
            const float2 f = s.found_at[w][i];
            own.key[j] = key_of(f.x), own.index[j] = __float_as_uint(f.y), own.weight[j] = weight_of(f.x, top, g.per_t);
        }
        part += own.weight[j];
    }
    if (g.by_k || g.by_p) {
        // (where there is no floor, what is 64 temperatures below the top and more shares the last bin, in which top-k may cut: with 32, 64 rows
        // of 600 logits took 28.1 us for 16.8, 16 of 300 24.7 for 17.8)
        const float spread = least_z > -INFINITY ? top - least_z : 64.f * g.t, per_bin = fminf((ROW_THREADS - 1) / spread, 3e38f);
        auto bin_of = [&](uint32_t key) { return bin_at(value_of(key), top, per_bin, ROW_THREADS); };
        empty_bins(c, tid);
        if (tid == 0) c.cut = nothing_cut();
        meet<NT>();
        fill_bins(own, c, bin_of);
        u64 whole = total;
        if (g.by_k) {
            const bool intact = find_cut<true>(own, c, (u64)g.top_k, top, per_bin);
            whole = c.cut.weight;
            if (g.by_p && !whole) {  // all are kept
                before_me<NT>(part, whole, c.sums);
                meet<NT>();  // (the waves' sums are written again by the next cut)
            }
            if (g.by_p && !intact) {
                meet<NT>();
                empty_bins(c, tid);
                meet<NT>();
                fill_bins(own, c, bin_of);
            }
        }
        if (g.by_p) find_cut<false>(own, c, max(share_of(g.top_p, whole, true), 1ull), top, per_bin);
    }
    // kept weights by index
    const Cut cut = g.by_k || g.by_p ? c.cut : nothing_cut();
    int left = 1 << 30;
    if (cut.some) {
        uint32_t ties = 0, all;
#pragma unroll
        for (int j = 0; j < OWN; ++j) ties += j < own.n && own.key[j] == cut.key;
        left = cut.ties - (int)before_me<NT>(ties, all, c.counts);
    }
    u64 w[OWN], all;
    part = 0;
#pragma unroll
    for (int j = 0; j < OWN; ++j) {
        const bool in = j < own.n && (double)top - (double)value_of(own.key[j]) <= reach && (own.key[j] == cut.key ? left-- > 0 : own.key[j] > cut.key);
        w[j] = in ? own.weight[j] : 0;
        part += w[j];
    }
    meet<NT>();
    u64 upto = before_me<NT>(part, all, c.sums);
    const u64 target = share_of(g.u, all, false);
    if (upto <= target && upto + part > target) {
        uint32_t token = 0xffffffffu;
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            upto += w[j];
            if (w[j] && upto > target) token = min(token, own.index[j]);
        }
        s.found = token;
    }
}

// Candidates are what may be kept: the tokens that are not below a floor which follows from the runs' numbers alone.
//   top-k  the floor is the k-th largest of the largest logits of runs of 64, or a little less: k tokens at least are not below it
//   top-p  tokens of a weight below (1 - p) * sum / vocab have less than (1 - p) * sum together, so that the others have p of it
//   min-p  its own
// A chain of dependent steps on one workgroup: with one cut 5 to 9 us, with top-k and top-p 11 to 16, of which the cuts take 6.
// They are few in most rows: read from the runs that have any, in the order of their indices, and held by one wave, or by all if they are
// more than 512: a wave alone needs no barriers (up to 512 of them: 2 us behind the loads, all eight waves 5).
template <typename T>
__global__ __launch_bounds__(ROW_THREADS) void sample_row_kernel(Sampling p, int third, char* shared_bins) {
    __shared__ RowShared s;
    constexpr int NT = ROW_THREADS;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = blockIdx.x;
    const T* z = (const T*)p.logits + (int64_t)r * p.row_stride;
    const SampleRow at(p.vocab);
    char* work = p.workspace + (size_t)r * at.bytes();
    const float* tops = (const float*)work;
    SampleNote* note = (SampleNote*)(work + at.note());
    const int n_chunks = at.runs * CHUNKS, per = (n_chunks + 4 * NT - 1) / (4 * NT);  // fours of chunks of a thread: 2 at most
    const Settings g(p, r);
    const bool scores = p.logprob || p.confidence;

    // the top, and the sums relative to it
    float chunk[8];
    float most = -INFINITY, low = INFINITY;
    bool nan = false;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int c = (tid * per + j) * 4;
        const float4 f = j < per && c < n_chunks ? *(const float4*)(tops + c) : float4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        chunk[4 * j] = f.x, chunk[4 * j + 1] = f.y, chunk[4 * j + 2] = f.z, chunk[4 * j + 3] = f.w;
        most = fmaxf(most, fmaxf(fmaxf(f.x, f.y), fmaxf(f.z, f.w)));
        nan |= f.x != f.x;  // (a run of 1024 with a NaN has sixteen)
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) low = chunk[j] > -INFINITY ? fminf(low, chunk[j]) : low;
    u64 sum = 0;
    float raw_run = 0, run_top = -INFINITY;
    if (tid < at.runs) {
        if (g.whole_sum()) sum = ((const u64*)(work + at.sums()))[tid];
        if (scores) raw_run = ((const float*)(work + at.raws()))[tid];
        const float4* f = (const float4*)(tops + tid * CHUNKS);
#pragma unroll
        for (int j = 0; j < CHUNKS / 4; ++j) run_top = fmaxf(run_top, fmaxf(fmaxf(f[j].x, f[j].y), fmaxf(f[j].z, f[j].w)));
    }
    const uint32_t wave_top = wave_most(nan ? 0xffffffffu : key_of(most)), wave_low = ~wave_most(~key_of(low));
    if (lane == 0) s.tops[wave] = wave_top, s.lows[wave] = wave_low;
    s.floor_count[tid] = 0;
    if (tid == 0) s.place = 0xffffffffu, s.found = 0xffffffffu, s.candidates = 0, s.floor_bin = NT, note->wide = 0;
    __syncthreads();
    uint32_t top_key = s.tops[0], low_key = s.lows[0];
    for (int i = 1; i < ROW_WAVES; ++i) top_key = max(top_key, s.tops[i]), low_key = min(low_key, s.lows[i]);
    if (g.bad || top_key >= KEY_INF || top_key <= KEY_NINF) {
        if (tid == 0) {
            p.token[r] = -1;
            if (p.logprob) p.logprob[r] = -INFINITY;
            if (p.confidence) p.confidence[r] = 0.f;
        }
        return;
    }
    const float top = value_of(top_key);
    const float run_ref = fmaxf(run_top, -MOST_FLOAT);
    double raw = 0;
    if (wave < (at.runs + 63) / 64) {
        if (g.whole_sum()) sum = rescaled(sum, ((double)run_ref - (double)top) * g.per_t);
        if (scores) {
            raw = wave_total((double)raw_run * power_of(((double)run_ref - (double)top) * 1.4426950408889634, 0));
        }
    }
    if (lane == 0) s.raw[wave] = raw;
    // bins for top-k's floor, between the largest and the least of the runs' largest
    const bool by_floor = g.by_k && g.top_k <= n_chunks;
    const float floor_per_bin = fminf((NT - 1) / (top - value_of(low_key)), 3e38f);
    if (by_floor) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (chunk[j] > -INFINITY) atomicAdd(&s.floor_count[bin_at(chunk[j], top, floor_per_bin, NT)], 1u);
    }
    u64 total;
    const u64 sum_before = before_me<NT>(sum, total, s.sums);
    raw = 0;
    for (int i = 0; i < (RUNS + 63) / 64; ++i) raw += s.raw[i];
    if (scores && wave == ROW_WAVES - 1) {
        const double l = log(raw);
        if (lane == 0) s.log_raw = l;
    }

    if (g.greedy) {
        // the first chunk that has it, the first in the chunk
#pragma unroll
        for (int j = 7; j >= 0; --j)
            if (j < 4 * per && chunk[j] == top) atomicMin(&s.place, tid * per * 4 + j);
        __syncthreads();
        if (wave == 0) {
            const int i = s.place * SAMPLE_CHUNK + lane;
            const u64 equal = __ballot(i < p.vocab && (float)z[min(i, p.vocab - 1)] == top);
            if (lane == 0) s.found = s.place * SAMPLE_CHUNK + __builtin_ctzll(equal);
        }
    } else if (!g.by_k && !g.by_p && !g.by_m) {
        // the run in which u * total lies, then the token in it, by the run's own weights
        const u64 target = share_of(g.u, total, false);
        if (sum_before <= target && sum_before + sum > target) s.place = tid, s.left = target - sum_before, s.ref = run_ref;
        __syncthreads();
        const int i = s.place * SAMPLE_RUN + tid * 2;
        const u64 left = s.left;
        const float ref = s.ref;
        const u64 w0 = i < p.vocab ? weight_of((float)z[i], ref, g.per_t) : 0, w1 = i + 1 < p.vocab ? weight_of((float)z[i + 1], ref, g.per_t) : 0;
        u64 all;
        const u64 before = before_me<NT>(w0 + w1, all, s.sums);
        const double y = ((double)ref - (double)top) * g.per_t;
        if (rescaled(before, y) <= left && rescaled(before + w0 + w1, y) > left) s.found = rescaled(before + w0, y) > left ? i : i + 1;
    } else {
        const double reach = g.by_m ? -log((double)g.min_p) * (double)g.t : INFINITY;
        uint32_t least = KEY_NINF;  // the floor's key
        if (by_floor) {
            const uint32_t c = s.floor_count[tid];
            uint32_t all;
            const uint32_t c_before = before_me<NT>(c, all, s.floors);
            if (c_before < (uint32_t)g.top_k && c_before + c >= (uint32_t)g.top_k) s.floor_bin = tid;
            __syncthreads();
            // (what is in these bins is above this, whatever the roundings; fewer than k runs with any: no floor)
            const int b = s.floor_bin;
            if (b < NT - 1) least = key_of(top - (float)(b + 1) / floor_per_bin * 1.00001f - fabsf(top) * 1e-6f);
        } else if (g.by_p && !g.by_k) {
            // (weights are off by less than one: what is below the floor's in full may be one above it as a whole number)
            const double floor_weight = (1.0 - (double)g.top_p) * (double)total / p.vocab * 0.99 - 1.0;
            if (floor_weight > 1.0) least = max(least, key_of((float)((double)top + log(floor_weight * 0x1p-44) * (double)g.t - fabs((double)top) * 1e-6)));
        }
        // (with both, top-p's share is of all of the first top_k, whatever min-p takes from them)
        if (g.by_m && !(g.by_k && g.by_p)) least = max(least, key_of((float)((double)top - reach - (fabs((double)top) + reach) * 1e-6)));
        least = min(least, top_key);
        const float least_z = value_of(least);

        // the runs that have candidates, in order
        uint32_t flags = 0, n_some;
#pragma unroll
        for (int j = 0; j < 8; ++j) flags |= (uint32_t)(chunk[j] >= least_z && chunk[j] > -INFINITY) << j;
        uint32_t place = before_me<NT>((uint32_t)__popc(flags), n_some, s.places);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (flags >> j & 1) s.chunks[place++] = (uint16_t)(tid * per * 4 + j);
        __syncthreads();
        // Tokens that lie anywhere leave exp(-n / chunks) of the runs without one: where this says that they are many more than can be
        // held, they are not looked for.
        bool wide = third && (float)n_some > (float)n_chunks * (1.f - __expf(-1.25f * CANDIDATES / (float)n_chunks));
        uint32_t n = 0;
        uint32_t from[ROW_WAVES];
        if (!wide) {
            // a wave takes neighbouring ones and keeps what it finds in its own place
            const int each = ((int)n_some + ROW_WAVES - 1) / ROW_WAVES, c0 = min((int)n_some, wave * each), c1 = min((int)n_some, c0 + each);
            uint32_t found = 0;
            const float from_z = fmaxf(least_z, -MOST_FLOAT);  // (nothing that is -inf)
            float next[AT_ONCE / 4][4];
            int next_at[AT_ONCE / 4];
            auto load = [&](int c) {  // sixteen lanes a chunk, so that the lanes' order is that of the indices
#pragma unroll
                for (int j = 0; j < AT_ONCE / 4; ++j) {
                    const int mine = c + 4 * j + (lane >> 4);
                    next_at[j] = s.chunks[min(mine, c1 - 1)] * SAMPLE_CHUNK + (lane & 15) * 4;
                    load4(z, mine < c1 ? next_at[j] : p.vocab, p.vocab, p.vec, next[j]);
                }
            };
            if (c0 < c1) load(c0);
            for (int c = c0; c < c1; c += AT_ONCE) {
                float v[AT_ONCE / 4][4];
                int at_index[AT_ONCE / 4];
#pragma unroll
                for (int j = 0; j < AT_ONCE / 4; ++j) {
                    at_index[j] = next_at[j];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[j][k] = next[j][k];
                }
                if (c + AT_ONCE < c1) load(c + AT_ONCE);
                const uint32_t found_before = found;
#pragma unroll
                for (int j = 0; j < AT_ONCE / 4; j += 2) {  // (two counts of 256 at most in a number)
                    uint32_t n = 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) n += (v[j][k] >= from_z ? 1u : 0u) + (v[j + 1][k] >= from_z ? 0x10000u : 0u);
                    const uint32_t upto = wave_scan(n), total_n = last_lane(upto), before = upto - n;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t slot = found + (h ? before >> 16 : before & 0xffff);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (v[j + h][k] >= from_z) {
                                if (slot < WAVE_CANDIDATES) s.found_at[wave][slot] = float2{v[j + h][k], __int_as_float(at_index[j + h] + k)};
                                ++slot;
                            }
                        found += h ? total_n >> 16 : total_n & 0xffff;
                    }
                }
                if (c + AT_ONCE < c1) {  // (too many already: the rest need not be read)
                    uint32_t all = 0;
                    if (lane == 0) all = atomicAdd(&s.candidates, found - found_before) + found - found_before;
                    if ((uint32_t)__builtin_amdgcn_readfirstlane((int)all) > CANDIDATES) {
                        found = WAVE_CANDIDATES + 1;
                        break;
                    }
                }
            }
            if (lane == 0) s.founds[wave] = found;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < ROW_WAVES; ++i) from[i] = n, n += s.founds[i], wide |= s.founds[i] > WAVE_CANDIDATES;
            wide |= n > CANDIDATES;
        }
        if (wide) {
            // (not without a third kernel: the host launches one wherever a row can have as many)
            if (!third) return;
            if (shared_bins) {
                u64* weights = (u64*)(shared_bins + (size_t)r * SAMPLE_ROW_BINS);
                uint32_t* counts = (uint32_t*)(weights + SAMPLE_BINS);
                for (int i = tid; i < SAMPLE_BINS; i += NT) weights[i] = 0, counts[i] = 0;
            }
            if (tid == 0) {
                note->top_key = top_key, note->least = least, note->arrived = 0, note->total = total, note->raw = raw;
                note->log_raw = scores ? log(raw) : 0.0;
                note->wide = 1;
            }
            return;
        }
        if (n <= ONE_WAVE) {
            if (wave == 0) token_of<64, ONE_WAVE / 64>(g, s, s.one, from, (int)n, top, least_z, reach, total);
        } else {
            token_of<NT, CANDIDATES / NT>(g, s, s.all, from, (int)n, top, least_z, reach, total);
        }
    }
    __syncthreads();
    if (tid == 0) {
        const int token = (int)min(s.found, (uint32_t)p.vocab - 1);
        write_row(p, r, token, scores ? (float)z[token] : 0.f, top, raw, scores ? s.log_raw : 0.0);
    }
}

// ------------------------------------------------------------------------------------------------
// rows with many candidates
// ------------------------------------------------------------------------------------------------
constexpr int WIDE_THREADS = 256, WIDE_WAVES = WIDE_THREADS / 64;
constexpr int MOST_PARTS = 16;

// What a workgroup of the row leaves for the last one: for each bin the weight of the part's elements before it, and how many these
// are in a list of them by bins, as indices in the part.  It goes past the caches of the XCD, by agent-scope stores and loads of
// single values.
struct Part {
    u64* weight;
    uint32_t* first;  // [SAMPLE_BINS + 1]
    uint16_t* element;
    __device__ __forceinline__ Part(char* parts, int part_length, int i) {
        char* base = parts + (size_t)i * sample_part_bytes(part_length);
        weight = (u64*)base, first = (uint32_t*)(weight + SAMPLE_BINS), element = (uint16_t*)(first + SAMPLE_BINS + 4);
    }
};
template <typename T>
__device__ __forceinline__ void leave(T* p, T v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename T>
__device__ __forceinline__ T take(const T* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The row's elements that are not below the floor, of [i0, i1), i0 a multiple of 4.
template <typename T>
struct RowElements {
    static constexpr int AT_ONCE = 4;
    const T* z;
    int i0, i1, vec;
    float top, least;
    double per_t;
    char* left;  // by the parts, if there are several
    int parts, part_length;
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        each(least, INFINITY, f);
    }
    template <typename F>
    __device__ __forceinline__ void each(float lo, float hi, F f) const {
        lo = fmaxf(lo, least);
        constexpr int STEP = WIDE_THREADS * 4;
        float next[AT_ONCE][4];
        auto load = [&](int i) {
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) load4(z, i + k * STEP, i1, vec, next[k]);
        };
        int i = i0 + threadIdx.x * 4;
        if (i < i1) load(i);
        for (; i < i1; i += STEP * AT_ONCE) {
            float v[AT_ONCE][4];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[k][j] = next[k][j];
            if (i + STEP * AT_ONCE < i1) load(i + STEP * AT_ONCE);
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (v[k][j] >= lo && v[k][j] <= hi && i + k * STEP + j < i1)
                        f(key_of(v[k][j]), i + k * STEP + j, [&] { return weight_of(v[k][j], top, per_t); });
        }
    }
    template <typename S>
    __device__ __forceinline__ bool list(S& s, int bin) const {
        if (parts == 1) return false;
        const int tid = threadIdx.x, lane = tid & 63;
        // (every wave looks the parts' shares up, one in a lane)
        uint32_t first = 0, n = 0;
        if (lane < parts) {
            const Part part(left, part_length, lane);
            first = take(part.first + bin), n = take(part.first + bin + 1) - first;
        }
        const uint32_t upto = wave_scan<16>(n);
        const int all = (int)of_lane(upto, 15);
        int at_part = 0;
        for (int i = 1; i < parts; ++i) at_part = tid >= (int)of_lane(upto, i - 1) ? i : at_part;
        const uint32_t start = (uint32_t)__shfl((int)first, at_part), before = (uint32_t)__shfl((int)(upto - n), at_part);
        if (tid < all) {  // (LIST at most)
            const int i = at_part * part_length + take(Part(left, part_length, at_part).element + start + (tid - before));
            const float v = (float)z[i];
            s.list[tid] = key_of(v), s.list_index[tid] = i, s.list_weight[tid] = weight_of(v, top, per_t);
        }
        if (tid == 0) s.n_list = all;
        return true;
    }
};
static_assert(LIST <= WIDE_THREADS, "a thread takes one element of a list");

struct WideShared {
    CutShared<WIDE_THREADS, SAMPLE_BINS> c;
    uint32_t last, found;
    int place, ties_left;
    u64 left;
    u64 part_weight[MOST_PARTS];
    uint32_t part_ties[MOST_PARTS];
    u64 run_weight[RUNS];
    uint32_t run_ties[RUNS];
};

// The bins of a row are filled by `parts` workgroups, and whoever is the last goes on: the cuts; the part of the row in which u * total
// lies, by the weights before the cut's bin in each part and the elements of that bin; the run of 1024 tokens, by the sums of what is
// kept in the part's runs; the token in it.  All sums are of whole numbers, so that their order does not matter.  One CU reads a
// row of 50 304 in 10 us (its loads wait for one another, see load4), so that nothing but the part's runs is read twice: unless the cut's bin has
// more than 256 elements, of which there is no list, as among many equal logits (4 rows of 200 000 in bf16 with top_k 30 000: 426 us).  22 to 30 us: bins 7, lists 5, cuts 4 each, the token 5.
template <typename T>
__global__ __launch_bounds__(WIDE_THREADS) void sample_wide_kernel(Sampling p, int parts, char* shared_bins, char* shared_parts) {
    __shared__ WideShared s;
    constexpr int NT = WIDE_THREADS, PER = SAMPLE_BINS / NT;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = blockIdx.x / parts, part = blockIdx.x % parts;
    const SampleRow at(p.vocab);
    SampleNote* note = (SampleNote*)(p.workspace + (size_t)r * at.bytes() + at.note());
    if (!note->wide) return;
    const T* z = (const T*)p.logits + (int64_t)r * p.row_stride;
    const Settings g(p, r);
    const float top = value_of(note->top_key), least_z = value_of(note->least);
    const float spread = note->least > KEY_NINF ? top - least_z : 32.f * g.t, per_bin = fminf((SAMPLE_BINS - 1) / spread, 3e38f);
    auto bin_of = [&](uint32_t key) { return bin_at(value_of(key), top, per_bin, SAMPLE_BINS); };

    empty_bins(s.c, tid);
    if (tid == 0) s.c.cut = nothing_cut(), s.found = 0xffffffffu, s.place = 0, s.left = 0, s.ties_left = 0;
    if (tid < MOST_PARTS) s.part_weight[tid] = 0, s.part_ties[tid] = 0;
    __syncthreads();
    const int runs_each = (at.runs + parts - 1) / parts, part_length = runs_each * SAMPLE_RUN;
    char* left = shared_parts + (size_t)r * parts * sample_part_bytes(part_length);
    const RowElements<T> own{z, part * part_length, min(p.vocab, (part + 1) * part_length), p.vec, top, least_z, g.per_t, left, parts, part_length};
    fill_bins(own, s.c, bin_of);
    if (parts > 1) {
        const Part here(left, part_length, part);
        u64* weights = (u64*)(shared_bins + (size_t)r * SAMPLE_ROW_BINS);
        uint32_t* counts = (uint32_t*)(weights + SAMPLE_BINS);
        uint32_t c[PER], c_all = 0, n;
        u64 w[PER], w_all = 0, all;
#pragma unroll
        for (int i = 0; i < PER; ++i) c[i] = s.c.bin_count[tid * PER + i], w[i] = s.c.bin_weight[tid * PER + i], c_all += c[i], w_all += w[i];
        uint32_t first = before_me<NT>(c_all, n, s.c.counts);
        u64 weight = before_me<NT>(w_all, all, s.c.sums);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int b = tid * PER + i;
            if (c[i]) {
                __hip_atomic_fetch_add(weights + b, w[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __hip_atomic_fetch_add(counts + b, c[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            leave(here.weight + b, weight);
            leave(here.first + b, first);
            s.c.bin_count[b] = first;  // (where the next of the bin's elements goes)
            first += c[i], weight += w[i];
        }
        if (tid == 0) leave(here.first + SAMPLE_BINS, n);
        __syncthreads();
        own.each([&](uint32_t key, int i, auto) { leave(here.element + atomicAdd(&s.c.bin_count[bin_of(key)], 1u), (uint16_t)(i - part * part_length)); });
        // what each thread has sent has arrived before its workgroup is counted
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) s.last = __hip_atomic_fetch_add(&note->arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)parts - 1;
        __syncthreads();
        if (!s.last) return;
#pragma unroll
        for (int i = 0; i < PER; ++i) w[i] = take(weights + tid * PER + i), c[i] = take(counts + tid * PER + i);
#pragma unroll
        for (int i = 0; i < PER; ++i) s.c.bin_weight[tid * PER + i] = w[i], s.c.bin_count[tid * PER + i] = c[i];
        __syncthreads();
    }
    const RowElements<T> row{z, 0, p.vocab, p.vec, top, least_z, g.per_t, left, parts, part_length};
    u64 whole = note->total;
    bool intact = true;  // (the bins by distance)
    if (g.by_k) {
        intact = find_cut<true>(row, s.c, (u64)g.top_k, top, per_bin);
        // (with top-p it does cut: the floor is top-k's alone then, and the bins hold what is not below it, top_k tokens at least, or all of
        // the row, the masked ones too)
        whole = s.c.cut.weight;
        if (g.by_p && !intact) {
            __syncthreads();
            empty_bins(s.c, tid);
            __syncthreads();
            fill_bins(row, s.c, bin_of);
        }
    }
    if (g.by_p) intact = find_cut<false>(row, s.c, max(share_of(g.top_p, whole, true), 1ull), top, per_bin);
    __syncthreads();
    Cut cut = s.c.cut;
    bool listed = (g.by_k || g.by_p) && s.c.listed;
    if (g.by_m) {  // cuts below the least key that is within reach
        const double reach = -log((double)g.min_p) * (double)g.t;
        auto within = [&](uint32_t key) { return (double)top - (double)value_of(key) <= reach; };
        uint32_t key = KEY_NINF + 1, high = note->top_key;  // (which is within it)
        while (key < high) {
            const uint32_t mid = key + (high - key) / 2;
            if (within(mid)) high = mid;
            else key = mid + 1;
        }
        if (key > cut.key) {  // (also where the other cut's own elements are the first out of reach)
            cut = Cut{key - 1, 0, 1, 0};
            const int bin = bin_of(cut.key);
            __syncthreads();  // (the list of another bin is read no more)
            listed = intact && s.c.bin_count[bin] <= LIST && row.list(s.c, bin);
            __syncthreads();
        }
    }
    auto kept_weight = [&](float v, uint32_t key) { return key > cut.key ? weight_of(v, top, g.per_t) : 0; };
    const u64 tie = cut.key && cut.ties ? weight_of(value_of(cut.key), top, g.per_t) : 0;
    // The part: what is kept in the bins before the cut's is all of them, in the cut's bin those of the list that are.  Where there is no
    // list (or nothing is cut), all of the row is one part.
    int first_run = 0, n_runs = at.runs, ties_before = 0;
    u64 target;
    const bool by_parts = parts > 1 && cut.key && listed;
    if (by_parts) {
        if (tid < (int)s.c.n_list) {
            const int at_part = (int)s.c.list_index[tid] / part_length;
            if (s.c.list[tid] == cut.key) atomicAdd(&s.part_ties[at_part], 1u);
            else if (s.c.list[tid] > cut.key) atomicAdd(&s.part_weight[at_part], s.c.list_weight[tid]);
        }
        const u64 before_bin = lane < parts ? take(Part(left, part_length, lane).weight + bin_of(cut.key)) : 0;
        __syncthreads();
        // (every wave for itself, a part in a lane)
        const uint32_t ties = lane < MOST_PARTS ? s.part_ties[lane] : 0;
        const int ties_left = max(0, cut.ties - (int)(wave_scan<16>(ties) - ties));
        const u64 w = before_bin + (lane < MOST_PARTS ? s.part_weight[lane] : 0) + tie * (u64)min((int)ties, ties_left);
        const u64 upto = wave_scan<16>(w);
        target = share_of(g.u, of_lane(upto, 15), false);
        const int at_part = __builtin_ctzll(__ballot(lane < MOST_PARTS && upto > target));
        target -= of_lane(upto - w, at_part);
        ties_before = cut.ties - __builtin_amdgcn_readlane(ties_left, at_part);
        first_run = at_part * runs_each, n_runs = min(runs_each, at.runs - first_run);
    }
    float v[4][4];
    auto load = [&](int run) {
#pragma unroll
        for (int k = 0; k < 4; ++k) load4(z, run * SAMPLE_RUN + k * 256 + lane * 4, p.vocab, p.vec, v[k]);
    };
    for (int run = wave; run < n_runs; run += WIDE_WAVES) {
        u64 w = 0;
        uint32_t ties = 0;
        load(first_run + run);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t key = key_of(v[k][j]);
                if (key == cut.key) ++ties;
                else w += kept_weight(v[k][j], key);
            }
        w = wave_scan(w), ties = wave_scan(ties);
        if (lane == 63) s.run_weight[run] = w, s.run_ties[run] = ties;
    }
    __syncthreads();
    {
        const uint32_t ties = tid < n_runs ? s.run_ties[tid] : 0;  // (RUNS <= WIDE_THREADS)
        uint32_t all_ties;
        u64 all;
        const int ties_left = max(0, cut.ties - ties_before - (int)before_me<NT>(ties, all_ties, s.c.counts));
        const u64 w = (tid < n_runs ? s.run_weight[tid] : 0) + tie * (u64)min((int)ties, ties_left);
        const u64 before = before_me<NT>(w, all, s.c.sums);
        if (!by_parts) target = share_of(g.u, all, false);
        if (before <= target && before + w > target) s.place = tid, s.left = target - before, s.ties_left = ties_left;
        __syncthreads();
    }
    if (s.place % WIDE_WAVES == wave) {
        load(first_run + s.place);
        u64 left = s.left;
        int ties_left = s.ties_left;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t ties = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) ties += key_of(v[k][j]) == cut.key;
            const uint32_t ties_upto = wave_scan(ties);
            int mine_left = ties_left - (int)(ties_upto - ties);
            u64 w[4], mine = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t key = key_of(v[k][j]);
                w[j] = key == cut.key ? (mine_left-- > 0 ? tie : 0) : kept_weight(v[k][j], key);
                mine += w[j];
            }
            const u64 upto = wave_scan(mine), all = last_lane(upto);
            u64 sum = upto - mine;
            if (left < all && sum <= left && upto > left) {
                int j_at = -1;
#pragma unroll
                for (int j = 3; j >= 0; --j) {
                    u64 to = sum;
#pragma unroll
                    for (int i = 0; i <= j; ++i) to += w[i];
                    if (to > left) j_at = j;
                }
                s.found = (first_run + s.place) * SAMPLE_RUN + k * 256 + lane * 4 + j_at;
            }
            if (left < all) break;
            left -= all, ties_left -= (int)last_lane(ties_upto);
        }
    }
    __syncthreads();
    if (tid == 0) {
        const int token = (int)min(s.found, (uint32_t)p.vocab - 1);
        write_row(p, r, token, (float)z[token], top, note->raw, note->log_raw);
    }
}

}  // namespace

// Rows with many candidates take sixteen workgroups each, or so many fewer that each has two runs and that there are 2048.  (50 304 logits, ten sets of rows with settings
// of every kind: 1 row 34.1 us with eight of them, 29.5 with sixteen, 28.8 with 32; 64 rows 43.3, 39.2, 39.5.  256 rows 119 us with two,
// 79 with eight, 71 with sixteen; 512 rows 171 with one, 121 with four, 103 with eight.  Where every row has many candidates, 512 rows
// take 248 with one, 292 with four, 342 with eight.  16 rows of 9000 logits: 50.5 with one, 41.5 with five, 40.8 with nine; 64 of 4000 39.8
// with one, 41.4 with two.  An element is noted in 16 bits in its part.)
int sample_parts(int rows, int vocab) {
    const int runs = SampleRow(vocab).runs;
    if (runs <= 4 || rows > 1024) return 1;
    return std::max(std::min(std::min(MOST_PARTS, (runs + 1) / 2), 2048 / std::max(rows, 1)), (runs + 63) / 64);
}
static size_t bins_at(int rows, int vocab) { return (SampleRow(vocab).bytes() * rows + 255) / 256 * 256; }

// Whether rows may have more candidates than the second kernel takes.
static bool third_kernel(int vocab, bool cuts) { return cuts && vocab > WAVE_CANDIDATES; }

size_t sample_workspace(int rows, int vocab, bool cuts) {
    const int parts = third_kernel(vocab, cuts) ? sample_parts(rows, vocab) : 1, runs = SampleRow(vocab).runs;
    const size_t shared = parts > 1 ? SAMPLE_ROW_BINS + sample_part_bytes((runs + parts - 1) / parts * SAMPLE_RUN) * parts : 0;
    return bins_at(rows, vocab) + shared * rows;
}

template <typename T>
static void launch_typed(const Sampling& p, hipStream_t st) {
    const SampleRow at(p.vocab);
    // 8192 waves, a few more than the chip holds at once (7 a SIMD), or so many fewer that all have the same number of runs
    const int64_t runs = (int64_t)p.rows * at.runs, each = (runs + 8191) / 8192, waves = (runs + each - 1) / each;
    EE_LAUNCH(sample_runs_kernel<T>, dim3((int)((waves + 3) / 4)), dim3(256), st, p, (int)each);
    const bool third = third_kernel(p.vocab, p.cuts());
    const int parts = sample_parts(p.rows, p.vocab);
    char* bins = p.workspace + bins_at(p.rows, p.vocab);
    EE_LAUNCH(sample_row_kernel<T>, dim3(p.rows), dim3(ROW_THREADS), st, p, third, third && parts > 1 ? bins : nullptr);
    if (!third) return;
    EE_LAUNCH(sample_wide_kernel<T>, dim3(p.rows * parts), dim3(WIDE_THREADS), st, p, parts, bins, bins + SAMPLE_ROW_BINS * p.rows);
}

hipError_t launch_sample(const Sampling& p, hipStream_t st) {
    if (p.dtype == EE_BF16)
        launch_typed<__bf16>(p, st);
    else
        launch_typed<float>(p, st);
    return hipGetLastError();
}

}  // namespace ee
