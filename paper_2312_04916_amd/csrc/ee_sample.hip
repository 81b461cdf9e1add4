// Choosing tokens (ee_sample of ee.h): one kernel passes over the logits and leaves a few numbers of each run of tokens, a second one
// finds a row's token from them and from the few runs that matter.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ee_lanes.h"
#include "ee_launch.h"
#include "ee_sample.h"

namespace ee {

namespace {

typedef unsigned long long u64;

constexpr int THREADS = 1024, WAVES = THREADS / 64;  // of the second kernel
constexpr int BINS = 1024;
constexpr int LIST = 512;       // elements of a bin that are ranked one by one
constexpr int OWN = 8;          // candidates of a thread
constexpr int CANDIDATES = THREADS * OWN;
constexpr int SEGMENTS = 1024;  // of a row with more candidates: runs of 256 tokens
constexpr int ONE = 44;         // weights are multiples of 2^-44 of the largest: 2^18 of them stay below 2^62
constexpr int CHUNKS = SAMPLE_RUN / SAMPLE_CHUNK;

// Order of the floats as unsigned numbers; -0 counts as 0, NaN as the largest.
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);
    return z != z ? 0xffffffffu : b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
constexpr uint32_t KEY_INF = 0xff800000u, KEY_NINF = 0x007fffffu;

// 2^y for y <= 0 as mantissa and exponent.  In 64 bits: the place of u * total among the sums has to be found in runs of 2^18
// weights.  2^f on [-1/2, 1/2] is a polynomial through nine Chebyshev nodes, its constant term kept at 1 (error 2^-45).
__device__ __forceinline__ double power_of(double y, int& exponent) {
    y = fmax(y, -1000.0);
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
    exponent = (int)n;
    return fma(g, f, 1.0);
}
// exp((z - top) / temperature) as a whole number of 2^-44, with per_t = log2(e) / temperature; adding 2^52 rounds to one and leaves it in the
// low bits.
__device__ __forceinline__ u64 weight_of(float z, float top, double per_t) {
    int e;
    const double m = power_of(((double)z - (double)top) * per_t, e);
    return (u64)__double_as_longlong(ldexp(m, e + ONE) + 0x1p52) & ((1ull << 52) - 1);
}
// a sum of weights relative to `top` as one relative to another top, 2^y times as large
__device__ __forceinline__ u64 rescaled(u64 sum, double y) {
    int e;
    const double m = power_of(y, e);
    return y == 0 ? sum : (u64)rint(ldexp((double)sum * m, e));
}

__device__ __forceinline__ u64 shfl_xor64(u64 v, int d) { return (u64)__shfl_xor((long long)v, d); }
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

// Four neighbouring elements, -inf behind the row's end
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
// the pass over the logits: a wave per run of 1024 tokens
// ------------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void sample_runs_kernel(Sampling p) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), waves = gridDim.x * 4;
    const SampleRow at(p.vocab);
    const uint32_t all = (uint32_t)p.rows * at.runs;
    const bool scores = p.logprob || p.confidence;
    for (uint32_t i = wave; i < all; i += waves) {
        const int r = i / (uint32_t)at.runs, run = i - r * at.runs;
        const T* z = (const T*)p.logits + (int64_t)r * p.row_stride;
        float v[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) load4(z, run * SAMPLE_RUN + j * 256 + lane * 4, p.vocab, p.vec, v[j]);
        char* out = p.workspace + (size_t)r * at.bytes();
        const Settings s(p, r);
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
            for (int j = 0; j < 4; ++j) ((float*)out)[run * CHUNKS + j * 4 + (lane >> 4)] = top[j];
        }
        const float ref = fmaxf(most, -3.4028235e38f);
        if (s.whole_sum()) {
            u64 sum = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) sum += weight_of(v[j][k], ref, s.per_t);
            sum = wave_total(sum);
            if (lane == 0) ((u64*)(out + at.sums()))[run] = sum;
        }
        if (scores) {
            float part[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                part[j] = (__expf(v[j][0] - ref) + __expf(v[j][1] - ref)) + (__expf(v[j][2] - ref) + __expf(v[j][3] - ref));
            const float raw = wave_sum((part[0] + part[1]) + (part[2] + part[3]));
            if (lane == 0) ((float*)(out + at.raws()))[run] = raw;
        }
    }
}

// ------------------------------------------------------------------------------------------------
// a row's token
// ------------------------------------------------------------------------------------------------

// What has been found out about a row: kept are the elements above `key` and the first `ties` ones (by index) that equal it.
struct Cut {
    uint32_t key;
    int ties;
    u64 weight;  // of all that is kept
};

struct Shared {
    u64 sums[WAVES];
    double raw[WAVES];
    uint32_t counts[WAVES], tops[WAVES];
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
    int place, ties_left;
    u64 left;
    float ref;
    uint32_t chunks[(1 << 18) / SAMPLE_CHUNK];
    union {
        struct {
            uint32_t key[CANDIDATES], index[CANDIDATES];
        } candidates;
        struct {
            u64 weight[SEGMENTS];
            uint32_t ties[SEGMENTS];
        } segments;
    };
};

// Sums over the workgroup: exclusive prefix of each thread's value, and the total.  `waves` is free again after the next barrier.
template <typename T>
__device__ __forceinline__ T before_me(T v, T& total, T* waves) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T in = wave_scan(v);
    if (lane == 63) waves[wave] = in;
    __syncthreads();
    T before = in - v;
    total = 0;
    for (int i = 0; i < WAVES; ++i) {
        if (i < wave) before += waves[i];
        total += waves[i];
    }
    return before;
}

// The elements that a cut is looked for among: f(key, weight()) for a thread's.  The whole row, those above a floor ...
template <typename T>
struct RowElements {
    const T* z;
    int n, vec;
    float top, least;
    double per_t;
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        for (int i = threadIdx.x * 4; i < n; i += THREADS * 4) {
            float v[4];
            load4(z, i, n, vec, v);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (v[j] >= least && i + j < n) f(key_of(v[j]), [&] { return weight_of(v[j], top, per_t); });
        }
    }
};
// ... or candidates that the threads hold.
struct OwnElements {
    const uint32_t (&key)[OWN];
    const u64 (&weight)[OWN];
    int n;
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int j = 0; j < OWN; ++j)
            if (j < n) f(key[j], [&] { return weight[j]; });
    }
};

// The last element that is kept where elements are kept, in their order, as long as fewer than `limit` came before (BY_COUNT) or
// their weights' sum is below `limit`: the bin in which that happens, then its elements one by one, or finer bins if they are many.
// Bins share the distance to the top, `per_bin` to one, and then the keys that are in the bin, until it holds one key only.  If all
// are kept, the cut is left as it was.
template <bool BY_COUNT, typename E>
__device__ void find_cut(const E& elements, Shared& s, u64 limit, float top, float per_bin) {
    const int tid = threadIdx.x;
    uint32_t lo = 0, hi = 0;
    int shift = -1;  // -1: bins by distance
    u64 base_weight = 0;
    uint32_t base_count = 0;
    for (;;) {
        auto bin_of = [&](uint32_t key) {
            if (shift < 0) return (int)fminf((top - value_of(key)) * per_bin, (float)(BINS - 1));
            return key >= lo && key <= hi ? (int)((hi - key) >> shift) : -1;
        };
        __syncthreads();
        s.bin_weight[tid] = 0, s.bin_count[tid] = 0;
        __syncthreads();
        // (what lies furthest may be most of a row: it is counted apart, not at one place by all)
        uint32_t last_count = 0;
        u64 last_weight = 0;
        elements.each([&](uint32_t key, auto weight) {
            const int b = bin_of(key);
            if (b == BINS - 1) {
                ++last_count;
                if (!BY_COUNT) last_weight += weight();
            } else if (b >= 0) {
                atomicAdd(&s.bin_count[b], 1u);
                if (!BY_COUNT) atomicAdd(&s.bin_weight[b], weight());
            }
        });
        if (last_count) atomicAdd(&s.bin_count[BINS - 1], last_count);
        if (last_weight) atomicAdd(&s.bin_weight[BINS - 1], last_weight);
        __syncthreads();
        // (BINS == THREADS)
        const uint32_t c = s.bin_count[tid];
        const u64 w = s.bin_weight[tid];
        const uint32_t c_in = wave_scan(c);
        const u64 w_in = BY_COUNT ? 0 : wave_scan(w);
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
        if (bin < 0) return;  // all are kept
        base_count = s.base_count, base_weight = s.base_weight;
        const uint32_t in_bin = s.in_bin;
        uint32_t key_lo = 0xffffffffu, key_hi = 0;
        elements.each([&](uint32_t key, auto weight) {
            if (bin_of(key) == bin) {
                key_lo = min(key_lo, key), key_hi = max(key_hi, key);
                if (in_bin <= LIST) {
                    const int at = atomicAdd(&s.n_list, 1);
                    s.list[at] = key, s.list_weight[at] = BY_COUNT ? 0 : weight();
                }
            }
        });
        if (key_lo <= key_hi) atomicMin(&s.lo, key_lo), atomicMax(&s.hi, key_hi);
        __syncthreads();
        lo = s.lo, hi = s.hi;
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
                if (mine)  // (all of one key write the same)
                    s.cut = Cut{key, (int)(BY_COUNT ? limit - above : (limit - weight + each - 1) / each), 0};
            }
            __syncthreads();
            return;
        }
        if (lo == hi) {  // one key: so many of them
            if (tid == 0) {
                const u64 each = s.bin_weight[bin] / in_bin;
                s.cut = Cut{lo, (int)(BY_COUNT ? limit - base_count : (limit - base_weight + each - 1) / each), 0};
            }
            __syncthreads();
            return;
        }
        shift = max(0, 32 - __builtin_clz(hi - lo) - 10);
    }
}

// More candidates than the threads hold: the same over the whole row.  Sums by segments of 256 tokens, the segment in which u * total
// lies, the token in it.
template <typename T>
__device__ int token_of_row(const RowElements<T>& row, const Settings& g, double reach, Shared& s, float per_bin) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    double far = INFINITY;
    Cut cut;
    auto kept_weight = [&](float z, uint32_t key) {
        return key >= cut.key && (double)row.top - (double)z <= far ? weight_of(z, row.top, row.per_t) : 0;
    };
    auto sum_up = [&] {  // of what is kept, ties apart
        for (int seg = wave; seg * 256 < row.n; seg += WAVES) {
            float v[4];
            load4(row.z, (seg * 64 + lane) * 4, row.n, row.vec, v);
            u64 w = 0;
            uint32_t ties = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t key = key_of(v[j]);
                if (key == cut.key) ++ties;
                else w += kept_weight(v[j], key);
            }
            if (__ballot(w != 0)) w = wave_total(w);
            if (__ballot(ties != 0))
                for (int d = 1; d < 64; d *= 2) ties += __shfl_xor(ties, d);
            if (lane == 0) s.segments.weight[seg] = w, s.segments.ties[seg] = ties;
        }
        __syncthreads();
    };
    const int n_seg = (row.n + 255) / 256;  // (SEGMENTS == THREADS)
    u64 tie, w, before, sum;
    uint32_t ties, ties_before, all_ties;
    int ties_left;
    auto prefix = [&] {
        cut = s.cut;
        tie = cut.key ? kept_weight(value_of(cut.key), cut.key) : 0;
        sum_up();
        ties = tid < n_seg ? s.segments.ties[tid] : 0;
        ties_before = before_me(ties, all_ties, s.counts);
        ties_left = max(0, cut.ties - (int)ties_before);
        w = (tid < n_seg ? s.segments.weight[tid] : 0) + tie * (u64)min((int)ties, ties_left);
        before = before_me(w, sum, s.sums);
        __syncthreads();
    };
    if (g.by_k) find_cut<true>(row, s, (u64)g.top_k, row.top, per_bin);
    if (g.by_p) {
        prefix();  // (of the first top_k, whatever min-p takes from them)
        find_cut<false>(row, s, max(share_of(g.top_p, sum, true), 1ull), row.top, per_bin);
    }
    far = reach;
    prefix();
    const u64 target = share_of(g.u, sum, false);
    if (before <= target && before + w > target) s.place = tid, s.left = target - before, s.ties_left = ties_left;
    __syncthreads();
    int token = 0;
    if (wave == 0) {
        const int i0 = (s.place * 64 + lane) * 4;
        float v[4];
        load4(row.z, i0, row.n, row.vec, v);
        uint32_t n_ties = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) n_ties += key_of(v[j]) == cut.key;
        int left = s.ties_left - (int)(wave_scan(n_ties) - n_ties);
        u64 own[4], mine = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t key = key_of(v[j]);
            own[j] = key == cut.key ? (left-- > 0 ? tie : 0) : kept_weight(v[j], key);
            mine += own[j];
        }
        u64 upto = wave_scan(mine) - mine;
        int at = 1 << 30;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            upto += own[j];
            if (upto > s.left) at = min(at, i0 + j);
        }
        for (int d = 1; d < 64; d *= 2) at = min(at, __shfl_xor(at, d));
        token = at;
    }
    return token;  // (of the first wave)
}

// Candidates are what may be kept: the tokens that are not below a floor which follows from the runs' numbers alone.
//   top-k  the floor is the k-th largest of the largest logits of runs of 64, or a little less: k tokens at least are not below it
//   top-p  tokens of a weight below (1 - p) * sum / vocab have less than (1 - p) * sum together, so that the others have p of it
//   min-p  its own
// They are few in most rows: read from the runs that have any, in the order of their indices, and held by the threads, eight each.
template <typename T>
__global__ __launch_bounds__(THREADS) void sample_kernel(Sampling p) {
    __shared__ Shared s;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = blockIdx.x;
    const T* z = (const T*)p.logits + (int64_t)r * p.row_stride;
    const SampleRow at(p.vocab);
    const char* work = p.workspace + (size_t)r * at.bytes();
    const float* tops = (const float*)work;
    const int n_chunks = at.runs * CHUNKS, per = (n_chunks + THREADS - 1) / THREADS;  // (4 at most)
    const Settings g(p, r);
    const bool scores = p.logprob || p.confidence;

    // the top, and the sums relative to it
    float chunk[4];
    uint32_t top_key = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int c = tid * per + j;
        chunk[j] = j < per && c < n_chunks ? tops[c] : -INFINITY;
        top_key = max(top_key, key_of(chunk[j]));
    }
    u64 sum = 0;
    float raw_run = 0, run_top = -INFINITY;
    if (tid < at.runs) {
        if (g.whole_sum()) sum = ((const u64*)(work + at.sums()))[tid];
        if (scores) raw_run = ((const float*)(work + at.raws()))[tid];
        const float4* f = (const float4*)(tops + tid * CHUNKS);
#pragma unroll
        for (int j = 0; j < CHUNKS / 4; ++j) run_top = fmaxf(run_top, fmaxf(fmaxf(f[j].x, f[j].y), fmaxf(f[j].z, f[j].w)));
    }
    for (int d = 1; d < 64; d *= 2) top_key = max(top_key, (uint32_t)__shfl_xor((int)top_key, d));
    if (lane == 0) s.tops[wave] = top_key;
    s.bin_count[tid] = 0;
    if (tid == 0) s.cut = Cut{0, 1 << 30, 0}, s.place = 1 << 30, s.left = 0, s.hi = 0xffffffffu;
    __syncthreads();
    for (int i = 0; i < WAVES; ++i) top_key = max(top_key, s.tops[i]);
    if (g.bad || top_key >= KEY_INF || top_key <= KEY_NINF) {
        if (tid == 0) {
            p.token[r] = -1;
            if (p.logprob) p.logprob[r] = -INFINITY;
            if (p.confidence) p.confidence[r] = 0.f;
        }
        return;
    }
    const float top = value_of(top_key);
    const float run_ref = fmaxf(run_top, -3.4028235e38f);
    double raw = 0;
    if (wave < (at.runs + 63) / 64) {
        if (g.whole_sum()) sum = rescaled(sum, ((double)run_ref - (double)top) * g.per_t);
        if (scores) {
            int e;
            const double m = power_of(((double)run_ref - (double)top) * 1.4426950408889634, e);
            raw = ldexp((double)raw_run * m, e);
            for (int d = 1; d < 64; d *= 2) raw += __shfl_xor(raw, d);
        }
    }
    if (lane == 0) s.raw[wave] = raw;
    u64 total;
    const u64 sum_before = before_me(sum, total, s.sums);
    raw = 0;
    for (int i = 0; i < WAVES; ++i) raw += s.raw[i];

    int token = 0;  // (of the first wave, or of all)
    if (g.greedy) {
        // the first chunk that has it, the first in the chunk
#pragma unroll
        for (int j = 3; j >= 0; --j)
            if (j < per && chunk[j] == top) atomicMin(&s.place, tid * per + j);
        __syncthreads();
        const int i = s.place * SAMPLE_CHUNK + lane;
        const u64 equal = __ballot(i < p.vocab && (float)z[min(i, p.vocab - 1)] == top);
        token = s.place * SAMPLE_CHUNK + __builtin_ctzll(equal);
    } else if (!g.by_k && !g.by_p && !g.by_m) {
        // the run in which u * total lies, then the token in it, by the run's own weights
        const u64 target = share_of(g.u, total, false);
        if (sum_before <= target && sum_before + sum > target) s.place = tid, s.left = target - sum_before, s.ref = run_ref;
        __syncthreads();
        const int i = s.place * SAMPLE_RUN + tid;
        const u64 left = s.left;
        const float ref = s.ref;
        const u64 w = i < p.vocab ? weight_of((float)z[i], ref, g.per_t) : 0;
        u64 all;
        const u64 before = before_me(w, all, s.sums);
        if (tid == 0) s.hi = 0xffffffffu;
        __syncthreads();
        if (w && rescaled(before + w, ((double)ref - (double)top) * g.per_t) > left) atomicMin(&s.hi, (uint32_t)i);
        __syncthreads();
        token = (int)s.hi;
    } else {
        const double reach = g.by_m ? -log((double)g.min_p) * (double)g.t : INFINITY;
        uint32_t least = KEY_NINF;  // the floor's key
        if (g.by_k && g.top_k <= n_chunks) {
            // bins between the largest and the least of the runs' largest
            uint32_t low = KEY_INF;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (chunk[j] > -INFINITY) low = min(low, key_of(chunk[j]));
            for (int d = 1; d < 64; d *= 2) low = min(low, (uint32_t)__shfl_xor((int)low, d));
            if (lane == 0) s.counts[wave] = low;
            __syncthreads();
            for (int i = 0; i < WAVES; ++i) low = min(low, s.counts[i]);
            const float per_bin = fminf((BINS - 1) / (top - value_of(low)), 3e38f);
            int bin[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bin[j] = chunk[j] > -INFINITY ? (int)fminf((top - chunk[j]) * per_bin, (float)(BINS - 1)) : BINS;
                if (bin[j] < BINS) atomicAdd(&s.bin_count[bin[j]], 1u);
            }
            __syncthreads();
            const uint32_t c = s.bin_count[tid];
            uint32_t all;
            const uint32_t c_before = before_me(c, all, s.counts);
            if (tid == 0) s.bin = BINS, s.lo = KEY_INF;
            __syncthreads();
            if (c_before < (uint32_t)g.top_k && c_before + c >= (uint32_t)g.top_k) s.bin = tid;
            __syncthreads();
            if (s.bin < BINS) {  // (else fewer than k runs have any: no floor)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (bin[j] <= s.bin) atomicMin(&s.lo, key_of(chunk[j]));
                __syncthreads();
                least = s.lo;
            }
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
        for (int j = 0; j < 4; ++j) flags |= (uint32_t)(chunk[j] >= least_z && chunk[j] > -INFINITY) << j;
        __syncthreads();
        uint32_t place = before_me((uint32_t)__popc(flags), n_some, s.counts);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (flags >> j & 1) s.chunks[place++] = tid * per + j;
        __syncthreads();
        // a wave takes neighbouring ones, eight loads at a time: how many candidates, then where they go
        const int each = ((int)n_some + WAVES - 1) / WAVES, c0 = min((int)n_some, wave * each), c1 = min((int)n_some, c0 + each);
        constexpr int AT_ONCE = 8;
        float v[AT_ONCE];
        int first[AT_ONCE];
        auto load = [&](int c) {
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                first[j] = (int)s.chunks[max(0, min(c + j, c1 - 1))] * SAMPLE_CHUNK;
                const int i = first[j] + lane;
                v[j] = c + j < c1 && i < p.vocab ? (float)z[i] : -INFINITY;
            }
        };
        auto wanted = [&](float x) { return x >= least_z && x > -INFINITY; };
        uint32_t found = 0;
        for (int c = c0; c < c1; c += AT_ONCE) {
            load(c);
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) found += __popcll(__ballot(wanted(v[j])));
        }
        if (lane == 0) s.tops[wave] = found;
        __syncthreads();
        uint32_t n = 0, base = 0;
        for (int i = 0; i < WAVES; ++i) {
            if (i < wave) base += s.tops[i];
            n += s.tops[i];
        }
        if (n > CANDIDATES) {
            const RowElements<T> row{z, p.vocab, p.vec, top, least_z, g.per_t};
            const float spread = least > KEY_NINF ? top - least_z : 32.f * g.t;
            token = token_of_row(row, g, reach, s, fminf((BINS - 1) / spread, 3e38f));
        } else {
            uint32_t index[OWN], key[OWN], to = base;
            u64 weight[OWN];
            for (int c = c0; c < c1; c += AT_ONCE) {
                if (each > AT_ONCE) load(c);  // (else they are here still)
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) {
                    const u64 some = __ballot(wanted(v[j]));
                    if (wanted(v[j])) {
                        const uint32_t slot = to + __popcll(some & ((1ull << lane) - 1));
                        s.candidates.key[slot] = key_of(v[j]), s.candidates.index[slot] = first[j] + lane;
                    }
                    to += __popcll(some);
                }
            }
            __syncthreads();
            const int mine = ((int)n + THREADS - 1) / THREADS, at0 = tid * mine;
#pragma unroll
            for (int j = 0; j < OWN; ++j) {
                const bool ok = j < mine && at0 + j < (int)n;
                key[j] = ok ? s.candidates.key[at0 + j] : 0;
                index[j] = ok ? s.candidates.index[at0 + j] : 0xffffffffu;
                weight[j] = ok ? weight_of(value_of(key[j]), top, g.per_t) : 0;
            }
            const OwnElements own{key, weight, max(0, min(mine, (int)n - at0))};
            const float per_bin = fminf((BINS - 1) / (top - least_z), 3e38f);
            // kept weights by index
            auto kept = [&](const Cut& cut, double far, u64 (&w)[OWN]) {
                uint32_t ties = 0, all;
#pragma unroll
                for (int j = 0; j < OWN; ++j) ties += j < own.n && key[j] == cut.key;
                int left = cut.ties - (int)before_me(ties, all, s.counts);
                u64 part = 0;
#pragma unroll
                for (int j = 0; j < OWN; ++j) {
                    const bool in = j < own.n && (double)top - (double)value_of(key[j]) <= far && (key[j] == cut.key ? left-- > 0 : key[j] > cut.key);
                    w[j] = in ? weight[j] : 0;
                    part += w[j];
                }
                return part;
            };
            u64 w[OWN], upto;
            if (g.by_k) find_cut<true>(own, s, (u64)g.top_k, top, per_bin);
            if (g.by_p) {
                u64 limit_of = total;
                if (g.by_k) {
                    const u64 part = kept(s.cut, INFINITY, w);
                    before_me(part, limit_of, s.sums);
                }
                find_cut<false>(own, s, max(share_of(g.top_p, limit_of, true), 1ull), top, per_bin);
            }
            const u64 part = kept(s.cut, reach, w);
            u64 all;
            upto = before_me(part, all, s.sums);
            const u64 target = share_of(g.u, all, false);
            if (tid == 0) s.hi = 0xffffffffu;
            __syncthreads();
            if (upto <= target && upto + part > target) {
#pragma unroll
                for (int j = 0; j < OWN; ++j) {
                    upto += w[j];
                    if (upto > target) atomicMin(&s.hi, index[j]);
                }
            }
            __syncthreads();
            token = (int)s.hi;
        }
    }
    if (tid == 0) {
        token = max(0, min(token, p.vocab - 1));
        p.token[r] = token;
        if (p.logprob) p.logprob[r] = (float)((double)(float)z[token] - (double)top - log(raw));
        if (p.confidence) p.confidence[r] = (float)(1.0 / raw);
    }
}

}  // namespace

hipError_t launch_sample(const Sampling& p, hipStream_t st) {
    const int64_t waves = (int64_t)p.rows * SampleRow(p.vocab).runs;
    const int grid = (int)std::min<int64_t>((waves + 3) / 4, 256 * 8);
    if (p.dtype == EE_BF16) {
        EE_LAUNCH(sample_runs_kernel<__bf16>, dim3(grid), dim3(256), st, p);
        EE_LAUNCH(sample_kernel<__bf16>, dim3(p.rows), dim3(THREADS), st, p);
    } else {
        EE_LAUNCH(sample_runs_kernel<float>, dim3(grid), dim3(256), st, p);
        EE_LAUNCH(sample_kernel<float>, dim3(p.rows), dim3(THREADS), st, p);
    }
    return hipGetLastError();
}

}  // namespace ee
