// Choosing tokens (ee_sample of ee.h): a workgroup per row.
#include <hip/hip_runtime.h>

#include "ee_launch.h"
#include "ee_sample.h"

namespace ee {

namespace {

typedef unsigned long long u64;

constexpr int THREADS = 1024, WAVES = THREADS / 64;
constexpr int BINS = 1024;
constexpr int LIST = 512;       // elements of a bin that are ranked one by one
constexpr int SEGMENTS = 1024;  // of a row: runs of 64 * PER neighbouring elements, PER at least 4
constexpr int ONE = 44;         // weights are multiples of 2^-44 of the largest: 2^18 of them stay below 2^62

// Order of the floats as unsigned numbers; -0 counts as 0, NaN as the largest.
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);
    return z != z ? 0xffffffffu : b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
constexpr uint32_t KEY_INF = 0xff800000u, KEY_NINF = 0x007fffffu;

// exp((z - top) / temperature) as a whole number of 2^-44, with per_t = log2(e) / temperature.  In 64 bits: the place of u * total among
// the sums has to be found in runs of 2^18 weights.  2^f on [-1/2, 1/2] is a polynomial through ten Chebyshev nodes
// with its constant term kept at 1 (error 2^-45); adding 2^52 rounds to a whole number and leaves it in the low bits.
__device__ __forceinline__ u64 weight_of(float z, float top, double per_t) {
    const double y = fmax(((double)z - (double)top) * per_t, -100.0);
    const double n = rint(y), f = y - n;
    double g = 0x1.b63880a30e9ffp-24;
    g = fma(g, f, 0x1.63d136366db24p-20);
    g = fma(g, f, 0x1.ffcb9515a8016p-17);
    g = fma(g, f, 0x1.4308ac85aa947p-13);
    g = fma(g, f, 0x1.5d87fe86fe88ep-10);
    g = fma(g, f, 0x1.3b2ab7181b755p-7);
    g = fma(g, f, 0x1.c6b08d7047e52p-5);
    g = fma(g, f, 0x1.ebfbdff823cedp-3);
    g = fma(g, f, 0x1.62e42fefa39efp-1);
    const double w = ldexp(fma(g, f, 1.0), (int)n + ONE) + 0x1p52;
    return (u64)__double_as_longlong(w) & ((1ull << 52) - 1);
}

template <typename T>
__device__ __forceinline__ T shfl_xor64(T v, int d) {
    return (T)__shfl_xor((long long)v, d);
}
__device__ __forceinline__ u64 wave_total(u64 v) {
    for (int d = 1; d < 64; d *= 2) v += shfl_xor64(v, d);
    return v;
}
// inclusive sums in the lanes' order
template <typename T>
__device__ __forceinline__ T wave_scan(T v) {
    const int lane = threadIdx.x & 63;
    for (int d = 1; d < 64; d *= 2) {
        const T o = sizeof(T) == 8 ? (T)__shfl_up((long long)v, d) : (T)__shfl_up((int)v, d);
        if (lane >= d) v += o;
    }
    return v;
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

// What has been found out about a row: kept are the elements above `key` and the first `ties` ones (by index) that equal it.
struct Cut {
    uint32_t key;
    int ties;
    u64 weight;  // of all that is kept
};

struct Shared {
    u64 sums[WAVES];
    double raw[WAVES];
    uint32_t counts[WAVES];
    u64 bin_weight[BINS];
    uint32_t bin_count[BINS];
    uint32_t list[LIST];
    u64 list_weight[LIST];
    int n_list;
    uint32_t lo, hi;  // keys of the bin that is looked into
    int bin;
    u64 base_weight;
    uint32_t base_count, in_bin;
    Cut cut;
    u64 seg_weight[SEGMENTS];
    uint32_t seg_ties[SEGMENTS];
    int segment;
    int ties_left;
    u64 left;
};

template <typename T>
struct Row {
    static constexpr int PER = 16 / sizeof(T);
    const T* z;
    int n, vec;
    // f(index, value) for a wave's elements, PER neighbouring ones per lane and 64 * PER per wave at a time: segment s holds
    // [64 * PER * s, 64 * PER * (s + 1))
    __device__ __forceinline__ void load(int i, float (&v)[PER]) const {
        if (vec && i + PER <= n) {
            typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
            const u32x4 a = *(const u32x4*)(z + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 2) {
                    v[2 * j] = __uint_as_float(a[j] << 16);
                    v[2 * j + 1] = __uint_as_float(a[j] & 0xffff0000u);
                } else {
                    v[j] = __uint_as_float(a[j]);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < PER; ++j) v[j] = i + j < n ? (float)z[i + j] : -INFINITY;
        }
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        for (int i0 = threadIdx.x * PER; i0 < n; i0 += THREADS * PER) {
            float v[PER];
            load(i0, v);
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (i0 + j < n) f(i0 + j, v[j]);
        }
    }
};

// The last element that is kept where elements are kept, in their order, as long as fewer than `limit` came before (BY_COUNT) or
// their weights' sum is below `limit`: the bin in which that happens, then its elements one by one, or finer bins if they are many.
// A bin's share is of the distance to the top first, and then of the keys that are in it, until it holds one key only.
template <bool BY_COUNT, typename T>
__device__ void find_cut(const Row<T>& row, Shared& s, u64 limit, float top, double per_t, float per_bin) {
    const int tid = threadIdx.x;
    uint32_t lo = 0, hi = 0;
    int shift = -1;  // -1: bins by distance
    u64 base_weight = 0;
    uint32_t base_count = 0;
    for (;;) {
        auto bin_of = [&](float z, uint32_t key) {
            if (shift < 0) return (int)fminf((top - z) * per_bin, (float)(BINS - 1));
            return key >= lo && key <= hi ? (int)((hi - key) >> shift) : -1;
        };
        if (shift >= 0) {
            __syncthreads();
            s.bin_weight[tid] = 0, s.bin_count[tid] = 0;
            __syncthreads();
            row.each([&](int, float z) {
                const int b = bin_of(z, key_of(z));
                if (b >= 0) {
                    atomicAdd(&s.bin_count[b], 1u);
                    atomicAdd(&s.bin_weight[b], weight_of(z, top, per_t));
                }
            });
            __syncthreads();
        }
        // (BINS == THREADS)
        const uint32_t c = s.bin_count[tid];
        const u64 w = s.bin_weight[tid];
        const uint32_t c_in = wave_scan(c);
        const u64 w_in = wave_scan(w);
        if ((tid & 63) == 63) s.counts[tid >> 6] = c_in, s.sums[tid >> 6] = w_in;
        if (tid == 0) s.n_list = 0, s.lo = 0xffffffffu, s.hi = 0, s.bin = -1;
        __syncthreads();
        uint32_t c_before = base_count + c_in - c;
        u64 w_before = base_weight + w_in - w;
        for (int i = 0; i < (tid >> 6); ++i) c_before += s.counts[i], w_before += s.sums[i];
        // the bin in which the limit is reached
        const bool here = c && (BY_COUNT ? c_before < limit && c_before + c >= limit : w_before < limit && w_before + w >= limit);
        if (here) s.bin = tid, s.base_count = c_before, s.base_weight = w_before, s.in_bin = c;
        __syncthreads();
        const int bin = s.bin;
        if (bin < 0) {  // all are kept
            __syncthreads();
            return;
        }
        base_count = s.base_count, base_weight = s.base_weight;
        const uint32_t in_bin = s.in_bin;
        uint32_t key_lo = 0xffffffffu, key_hi = 0;
        row.each([&](int, float z) {
            const uint32_t key = key_of(z);
            if (bin_of(z, key) == bin) {
                key_lo = min(key_lo, key), key_hi = max(key_hi, key);
                if (in_bin <= LIST) {
                    const int at = atomicAdd(&s.n_list, 1);
                    s.list[at] = key, s.list_weight[at] = weight_of(z, top, per_t);
                }
            }
        });
        if (key_lo <= key_hi) atomicMin(&s.lo, key_lo), atomicMax(&s.hi, key_hi);
        __syncthreads();
        lo = s.lo, hi = s.hi;
        if (lo == hi) {  // one key: so many of them
            if (tid == 0) {
                const u64 each = weight_of(value_of(lo), top, per_t);
                const u64 ties = BY_COUNT ? limit - base_count : each ? (limit - base_weight + each - 1) / each : 1;
                s.cut = Cut{lo, (int)ties, base_weight + ties * each};
            }
            __syncthreads();
            return;
        }
        if (in_bin <= LIST) {
            const int n = s.n_list;
            if (tid < n) {
                const uint32_t key = s.list[tid];
                const u64 each = s.list_weight[tid];
                uint32_t above = base_count, equal = 0;
                u64 weight = base_weight;
                for (int i = 0; i < n; ++i) {
                    const uint32_t k = s.list[i];
                    if (k > key) ++above, weight += s.list_weight[i];
                    if (k == key) ++equal;
                }
                const bool mine = BY_COUNT ? above < limit && above + equal >= limit : weight < limit && weight + equal * each >= limit;
                if (mine) {  // (all of one key write the same)
                    const u64 ties = BY_COUNT ? limit - above : (limit - weight + each - 1) / each;
                    s.cut = Cut{key, (int)ties, weight + ties * each};
                }
            }
            __syncthreads();
            return;
        }
        const int bits = 32 - __builtin_clz(hi - lo);
        shift = max(0, bits - 10);
    }
}

// One row: its top and whether it has a distribution; the sums of the weights and of the exponentials of the logits as they are; where
// top-k and then top-p cut; the kept weights' sums by segments; the segment, then the token.
template <typename T>
__global__ __launch_bounds__(THREADS) void sample_kernel(Sampling p) {
    __shared__ Shared s;
    constexpr int PER = Row<T>::PER;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = blockIdx.x;
    const Row<T> row{(const T*)p.logits + (int64_t)r * p.row_stride, p.vocab, p.vec};
    const float u = p.u[r], t = p.temperature ? p.temperature[r] : p.one_temperature;
    const int top_k = p.top_k ? p.top_k[r] : p.one_top_k;
    const float top_p = p.top_p ? p.top_p[r] : p.one_top_p, min_p = p.min_p ? p.min_p[r] : p.one_min_p;
    const bool bad = !(u >= 0.f && u < 1.f) || !(t >= 0.f && t < INFINITY) || top_k < 0 || !(top_p >= 0.f && top_p <= 1.f) || !(min_p >= 0.f && min_p <= 1.f);

    u64 best = 0;  // key, then the lowest index
    row.each([&](int i, float z) { best = max(best, (u64)key_of(z) << 32 | (uint32_t)~i); });
    for (int d = 1; d < 64; d *= 2) best = max(best, shfl_xor64(best, d));
    if (lane == 0) s.sums[wave] = best;
    s.bin_weight[tid] = 0, s.bin_count[tid] = 0;
    __syncthreads();
    for (int i = 0; i < WAVES; ++i) best = max(best, s.sums[i]);
    const uint32_t top_key = (uint32_t)(best >> 32);
    if (bad || top_key >= KEY_INF || top_key <= KEY_NINF) {
        if (tid == 0) {
            p.token[r] = -1;
            if (p.logprob) p.logprob[r] = -INFINITY;
            if (p.confidence) p.confidence[r] = 0.f;
        }
        return;
    }
    const float top = value_of(top_key);
    const bool greedy = t == 0.f, scores = p.logprob || p.confidence;
    const bool by_k = !greedy && top_k > 0 && top_k < p.vocab, by_p = !greedy && top_p < 1.f, by_m = !greedy && min_p > 0.f;
    const double per_t = greedy ? 0.0 : 1.4426950408889634 / (double)t;
    const float per_bin = greedy ? 0.f : fminf(32.f / t, 3e38f);

    u64 total = 0;
    double raw = 0;
    row.each([&](int, float z) {
        if (scores) raw += (double)__expf(z - top);
        if (greedy) return;
        const u64 w = weight_of(z, top, per_t);
        total += w;
        if (by_k || by_p) {
            const int b = (int)fminf((top - z) * per_bin, (float)(BINS - 1));
            atomicAdd(&s.bin_count[b], 1u);
            atomicAdd(&s.bin_weight[b], w);
        }
    });
    total = wave_total(total);
    for (int d = 1; d < 64; d *= 2) raw += __shfl_xor(raw, d);
    __syncthreads();
    if (lane == 0) s.sums[wave] = total, s.raw[wave] = raw;
    if (tid == 0) s.cut = Cut{0, 1 << 30, 0};
    __syncthreads();
    total = 0, raw = 0;
    for (int i = 0; i < WAVES; ++i) total += s.sums[i], raw += s.raw[i];
    __syncthreads();

    int token = (int)~(uint32_t)best;
    if (!greedy) {
        if (by_k) {
            find_cut<true>(row, s, (u64)top_k, top, per_t, per_bin);
            total = s.cut.weight;
        }
        if (by_p) {
            if (by_k) {  // (the bins may have been finer ones)
                __syncthreads();
                s.bin_weight[tid] = 0, s.bin_count[tid] = 0;
                __syncthreads();
                row.each([&](int, float z) {
                    const int b = (int)fminf((top - z) * per_bin, (float)(BINS - 1));
                    atomicAdd(&s.bin_count[b], 1u);
                    atomicAdd(&s.bin_weight[b], weight_of(z, top, per_t));
                });
                __syncthreads();
            }
            find_cut<false>(row, s, max(share_of(top_p, total, true), 1ull), top, per_t, per_bin);
        }
        const Cut cut = s.cut;
        const double reach = by_m ? -log((double)min_p) * (double)t : INFINITY;
        auto kept_weight = [&](float z, uint32_t key) { return key >= cut.key && (double)top - (double)z <= reach ? weight_of(z, top, per_t) : 0; };
        const u64 tie = cut.key ? kept_weight(value_of(cut.key), cut.key) : 0;
        // by segments
        for (int seg = wave; seg * 64 * PER < p.vocab; seg += WAVES) {
            float v[PER];
            row.load((seg * 64 + lane) * PER, v);
            u64 w = 0;
            uint32_t ties = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const uint32_t key = key_of(v[j]);
                if (key == cut.key) ++ties;
                else w += kept_weight(v[j], key);
            }
            if (__ballot(w != 0)) w = wave_total(w);
            if (__ballot(ties != 0))
                for (int d = 1; d < 64; d *= 2) ties += __shfl_xor(ties, d);
            if (lane == 0) s.seg_weight[seg] = w, s.seg_ties[seg] = ties;
        }
        __syncthreads();
        const int n_seg = (p.vocab + 64 * PER - 1) / (64 * PER);
        // (SEGMENTS == THREADS)
        const uint32_t ties = tid < n_seg ? s.seg_ties[tid] : 0;
        uint32_t ties_in = wave_scan(ties);
        if (lane == 63) s.counts[wave] = ties_in;
        __syncthreads();
        for (int i = 0; i < wave; ++i) ties_in += s.counts[i];
        const int ties_left = max(0, cut.ties - (int)(ties_in - ties));
        const u64 w = (tid < n_seg ? s.seg_weight[tid] : 0) + tie * (u64)min((int)ties, ties_left);
        u64 w_in = wave_scan(w);
        if (lane == 63) s.sums[wave] = w_in;
        __syncthreads();
        for (int i = 0; i < wave; ++i) w_in += s.sums[i];
        u64 sum = 0;
        for (int i = 0; i < WAVES; ++i) sum += s.sums[i];
        const u64 target = share_of(u, sum, false);
        if (w_in > target && w_in - w <= target) s.segment = tid, s.left = target - (w_in - w), s.ties_left = ties_left;
        __syncthreads();
        if (wave == 0) {
            const int i0 = (s.segment * 64 + lane) * PER;
            float v[PER];
            row.load(i0, v);
            uint32_t n_ties = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) n_ties += key_of(v[j]) == cut.key;
            int left = s.ties_left - (int)(wave_scan(n_ties) - n_ties);
            u64 own[PER], mine = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const uint32_t key = key_of(v[j]);
                own[j] = key == cut.key ? (left-- > 0 ? tie : 0) : kept_weight(v[j], key);
                mine += own[j];
            }
            u64 before = wave_scan(mine) - mine;
            int at = 1 << 30;
#pragma unroll
            for (int j = PER - 1; j >= 0; --j) {
                u64 upto = before;
#pragma unroll
                for (int i = 0; i <= j; ++i) upto += own[i];
                if (upto > s.left) at = i0 + j;
            }
            for (int d = 1; d < 64; d *= 2) at = min(at, __shfl_xor(at, d));
            token = min(at, p.vocab - 1);
        }
    }
    if (tid == 0) {
        p.token[r] = token;
        if (p.logprob) p.logprob[r] = (float)((double)(float)row.z[token] - (double)top - log(raw));
        if (p.confidence) p.confidence[r] = (float)(1.0 / raw);
    }
}

}  // namespace

hipError_t launch_sample(const Sampling& p, hipStream_t st) {
    if (p.dtype == EE_BF16)
        EE_LAUNCH(sample_kernel<__bf16>, dim3(p.rows), dim3(THREADS), st, p);
    else
        EE_LAUNCH(sample_kernel<float>, dim3(p.rows), dim3(THREADS), st, p);
    return hipGetLastError();
}

}  // namespace ee
