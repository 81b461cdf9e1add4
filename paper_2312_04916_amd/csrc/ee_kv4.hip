// Kernels of the 4-bit paged cache: plan, append, read and attention (ee_kv4_* of ee.h; layouts in ee_kv4.h).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ee_kv4.h"
#include "ee_lanes.h"
#include "ee_launch.h"

namespace ee {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// x / d, with magic = magic_of(d): the multiplier 2^32 / d, rounded up, gives it or one more.
__device__ __forceinline__ uint32_t div_by(uint32_t x, uint32_t d, uint32_t magic) {
    if (d == 1) return x;
    const uint32_t q = __umulhi(x, magic);
    return q * d > x ? q - 1 : q;
}
// x / d for 0 <= x < 2^20, d > 0: the reciprocal's and the product's errors leave the quotient, or one beside it.
__device__ __forceinline__ int div_small(int x, int d) {
    int q = (int)((float)x * __builtin_amdgcn_rcpf((float)d));
    q -= q * d > x ? 1 : 0;
    return q + ((q + 1) * d <= x ? 1 : 0);
}

constexpr uint32_t SCALE_NAN = 255;              // of a group that stands for NaN
constexpr uint32_t SCALE_MIN = 16, SCALE_MAX = 252;  // 2^-111, 2^125: no held value is subnormal or infinite in bf16

// ------------------------------------------------------------------------------------------------
// create
// ------------------------------------------------------------------------------------------------
__global__ void kv4_init_kernel(int32_t* table, int64_t n_table, int32_t* free_blocks, int n_blocks, uint32_t* arrived, int n_arrived,
                                uint32_t* counts) {
    const int64_t i0 = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = i0; i < n_table; i += step) table[i] = 0;
    for (int64_t i = i0; i < n_blocks; i += step) free_blocks[i] = n_blocks - 1 - (int)i;  // block 0 is on top
    for (int64_t i = i0; i < n_arrived; i += step) arrived[i] = 0;
    if (i0 < 4) counts[i0] = i0 == 0 ? n_blocks : 0;
}

// ------------------------------------------------------------------------------------------------
// plan
// ------------------------------------------------------------------------------------------------
constexpr int PLAN_SEQS = EE_KV4_MAX_SEQS + 1;  // and the rows behind the last request's

// inclusive sums over a wave (over each of its rows of 16 lanes if ROWS), in the lanes' order
template <bool ROWS = false>
__device__ __forceinline__ int lanes_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // from the lane 1, 2, 4, 8 before in the row
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    if constexpr (!ROWS) {
        v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // the last of row 0, 2 to row 1, 3
        v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // the last of row 1 to rows 2 and 3
    }
    return v;
}

// largest of a wave's values, none of them negative
__device__ __forceinline__ int lanes_max(int v) {
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(v, 63);
}

// Sums over a workgroup of up to 16 waves: exclusive prefix of each thread's values, and the totals.  `waves` is used by one
// call only.
template <int N>
__device__ __forceinline__ void scan_sums(int (&v)[N], int (&total)[N], int (*waves)[N]) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n_waves = blockDim.x >> 6;
    int own[N];
#pragma unroll
    for (int k = 0; k < N; ++k) own[k] = v[k], v[k] = lanes_scan(v[k]);
    if (lane == 63) {
#pragma unroll
        for (int k = 0; k < N; ++k) waves[wave][k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int sums = lanes_scan<true>(lane < n_waves ? waves[lane][k] : 0);
        total[k] = __builtin_amdgcn_readlane(sums, 15);
        v[k] += (wave ? __builtin_amdgcn_readlane(sums, wave - 1) : 0) - own[k];
    }
}

// Last index i < n with first[i] <= x (first ascending, first[0] <= x): of several equal ones the last, which is the one that
// is not empty.
__device__ __forceinline__ int last_not_above(const int32_t* first, int n, int32_t x) {
    int lo = 0, len = n;  // (a step reads three places at once: LDS answers late, not slowly)
    while (len > 1) {
        const int q = (len + 3) >> 2, a = min(lo + q, lo + len - 1), b = min(lo + 2 * q, lo + len - 1), c = min(lo + 3 * q, lo + len - 1);
        const bool ga = first[a] <= x, gb = first[b] <= x, gc = first[c] <= x;
        const int end = gc ? lo + len : gb ? c : ga ? b : a;
        lo = gc ? c : gb ? b : ga ? a : lo;
        len = end - lo;
    }
    return lo;
}

// Blocks of a request: before ceil(held / B), after ceil(end / B); which ones go where follows from three running sums over the
// requests (given back, asked for, rows) and from which of them are served, which again is a running sum's comparison.
// Every workgroup forms the sums over all requests for itself (a few thousand lengths at most: cheaper than handing them on)
// and takes its share of what has to be written, one thread per row, block and part, which finds its request by a search in
// LDS.  What a workgroup reads, no other one writes: a block that one request gives back and another one takes is looked up in
// the table row of the first, behind what it keeps, which nothing changes; and held_next, which may be where the lengths are
// read, is written by the workgroup that is the last to have read them.  All sums fit 32 bits: a request has at most 2^16
// blocks, and a thread's rows are counted up to n_rows + 1, at most 2^20 + 1.
// Bound by latency: lengths, sums, search, table, store, one after the other.  16 requests with 38 rows 4.9 us, of which an empty
// launch is 3.5; 1000 requests with 6 800 rows 8.0 us; 200 that bring prompts of up to 2048 rows 8.3 us for 2.3 MB.
constexpr int SERVED = 1 << 30, BLOCKS = SERVED - 1;  // in s_had
__global__ __launch_bounds__(1024) void kv4_plan_kernel(Kv4Plan p) {
    __shared__ int32_t s_row[PLAN_SEQS + 1];    // first row
    __shared__ int32_t s_take[PLAN_SEQS + 1];   // blocks taken by the requests before
    __shared__ int32_t s_give[PLAN_SEQS + 1];   // blocks given back by the requests before
    __shared__ int32_t s_start[PLAN_SEQS + 1];  // first row's position
    __shared__ int32_t s_had[PLAN_SEQS + 1];    // blocks held before, SERVED
    __shared__ int32_t s_part[PLAN_SEQS + 1];   // first part, of requests and then of the rows behind them
    __shared__ int32_t s_slot[PLAN_SEQS + 1];   // first slot of parts that are joined
    __shared__ int s_sums[16][4], s_sums2[16][4], s_sums3[16][2];
    __shared__ float s_work[16];
    __shared__ int s_taken[16], s_last;
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 63, wave = tid >> 6;
    const int n = p.n_seqs, per = (n + nt) / nt;  // requests of a thread, with the one behind the last
    const int i0 = min(n, tid * per), i1 = min(n, i0 + per);
    const int most = p.max_positions, bt_shift = p.block_shift, bt = 1 << bt_shift, cap = p.n_rows + 1;
    const bool first_wg = blockIdx.x == 0;

    // lengths; blocks held, given back, asked for; rows
    int sum[4] = {0, 0, 0, 0}, all[4];
    for (int i = i0; i < i1; ++i) {
        const int held = p.held[i], start = p.start[i], end = p.end[i];
        const bool range = start >= 0 && start <= end && end <= most;
        const bool gap = start > held && start < end;  // (its rows would see positions that nobody has written)
        const bool ok = range && held >= 0 && held <= most && !gap && end - start <= p.max_rows_per_seq;
        const int had = (min(max(held, 0), most) + bt - 1) >> bt_shift, need = ok ? (end + bt - 1) >> bt_shift : had;
        const int rows = range ? min(end - start, cap) : 0;
        s_start[i] = start, s_had[i] = had | (ok ? SERVED : 0), s_take[i] = need, s_row[i] = rows;  // (this thread's, for now)
        sum[0] += had, sum[1] += max(had - need, 0), sum[2] += max(need - had, 0);
        sum[3] = min(sum[3] + rows, cap);
    }
    scan_sums<4>(sum, all, s_sums);
    uint32_t arrived = 0;  // (all of this workgroup's lengths have been read; the answer is needed at the end)
    if (tid == 0 && gridDim.x > 1) arrived = __hip_atomic_fetch_add(p.arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int left = max(0, p.n_blocks - all[0]);  // free before the call (the lengths may contradict the pool)
    const bool clipped = all[3] > p.n_rows;
    if (clipped) {
        // rows that do not fit: their requests are refused, and give and take nothing (no rows always fit: a request that ends
        // gives its blocks back)
        int row = sum[3], again[4] = {0, 0, 0, 0};
        for (int i = i0; i < i1; ++i) {
            const int rows = s_row[i];
            if (rows > 0 && row + rows > p.n_rows) s_had[i] &= BLOCKS, s_take[i] = s_had[i];
            const int had = s_had[i] & BLOCKS, need = s_take[i];
            again[1] += max(had - need, 0), again[2] += max(need - had, 0);
            row = min(row + rows, cap);
        }
        int all2[4];
        scan_sums<4>(again, all2, s_sums2);
        sum[1] = again[1], sum[2] = again[2], all[1] = all2[1], all[2] = all2[2];
    }
    const int given = all[1], have = left + given, rows_all = min(all[3], p.n_rows);

    // served; the work of the rows in chunks of positions per kv head
    float work = 0.f;
    int taken = 0;
    {
        int give = sum[1], take = sum[2], row = sum[3];
        for (int i = i0; i < i1; ++i) {
            const int had = s_had[i] & BLOCKS, need = s_take[i], rows = s_row[i], asked = max(need - had, 0);
            const bool ok = (s_had[i] & SERVED) && (asked == 0 || take + asked <= have);
            const int row0 = min(row, p.n_rows), row1 = min(row + rows, p.n_rows);
            s_row[i] = row0, s_take[i] = min(take, have), s_give[i] = give, s_had[i] = had | (ok ? SERVED : 0);
            give += max(had - need, 0), take += asked, row = min(row + rows, cap);
            if (ok) {
                if (asked) taken = take;
                if (row1 > row0) {
                    const int tiles = ((row1 - row0) * p.group + p.tile_rows - 1) >> p.tile_shift;
                    work += (float)tiles * (float)((s_start[i] + row1 - row0 + KV4_CHUNK - 1) / KV4_CHUNK);
                }
            }
            if (first_wg) p.a.served[i] = ok ? 1 : 0, p.a.row_start[i] = row0;
        }
        if (tid == 0) s_row[n] = rows_all, s_row[n + 1] = p.n_rows, s_give[n] = given;
    }
    work = wave_sum(work);
    taken = lanes_max(taken);
    if (lane == 0) s_work[wave] = work, s_taken[wave] = taken;
    __syncthreads();
    work = wave_sum(lane < nt >> 6 ? s_work[lane] : 0.f);
    taken = lanes_max(lane < nt >> 6 ? s_taken[lane] : 0);
    // chunks of a part: an even share of the work.  Where the parts all run at once, more of them would run after the others have
    // ended: an item is cut into as many parts as it has shares, three quarters of one counting (17 requests of 500 to 12 560
    // positions, 32 heads on 8: 15 rows each 61 us, 1 to 15 rows 44; with whole shares only, and parts of nearly two, 68 and 44;
    // with halves counting too, 66 and 52).  Else into one more, so that none is longer than a share.
    const int per_part = max(p.min_chunks, (int)fminf(65536.f, ceilf(work * (float)p.kv_heads / (float)p.target_parts)));
    const int round_up = p.whole_shares ? per_part / 4 : per_part - 1;

    // parts: items (tile of rows, kv head) in the requests' order, each cut alike; the rows behind the last request's are one
    // more request that sees nothing
    auto parts_of = [&](int i) {  // of an item
        const int rows = s_row[i + 1] - s_row[i];
        if (i == n || rows == 0 || !(s_had[i] & SERVED)) return 1;
        return max(1, div_small(min((s_start[i] + rows + KV4_CHUNK - 1) / KV4_CHUNK + round_up, (1 << 20) - 1), per_part));
    };
    auto items_of = [&](int i) { return (((s_row[i + 1] - s_row[i]) * p.group + p.tile_rows - 1) >> p.tile_shift) * p.kv_heads; };
    int cnt[2] = {0, 0}, cnt_all[2];
    const int j0 = min(n + 1, tid * per), j1 = min(n + 1, j0 + per);
    for (int i = j0; i < j1; ++i) {
        const int np = parts_of(i), all_parts = items_of(i) * np;
        s_part[i] = all_parts, s_slot[i] = np;  // (this thread's, for now)
        cnt[0] += all_parts, cnt[1] += np > 1 ? all_parts : 0;
    }
    scan_sums<2>(cnt, cnt_all, s_sums3);
    for (int i = j0; i < j1; ++i) {
        const int all_parts = s_part[i], np = s_slot[i];
        s_part[i] = cnt[0], s_slot[i] = cnt[1];
        cnt[0] += all_parts, cnt[1] += np > 1 ? all_parts : 0;
    }
    __syncthreads();
    const int n_parts = min(cnt_all[0], p.max_parts);
    if (first_wg && tid == 0) p.counts[0] = n_parts, p.counts[1] = p.shape, *p.a.n_free = have - taken, p.a.row_start[n] = rows_all;

    // entry `at` of the stack as it stands once everything given back lies on it
    auto stack = [&](int at) {
        if (at < left) return p.a.free_blocks[at];
        const int back = given - 1 - (at - left);  // in the requests' order, first block first
        const int i = last_not_above(s_give, n, back);
        const int need = (s_had[i] & BLOCKS) - (s_give[i + 1] - s_give[i]);
        return p.a.table[(size_t)i * p.table_stride + min(need + back - s_give[i], p.table_stride - 1)];
    };
    const int64_t n_tasks = (int64_t)p.n_rows + taken + given + n_parts;
    for (int64_t task = (int64_t)blockIdx.x * nt + tid; task < n_tasks; task += (int64_t)gridDim.x * nt) {
        int64_t t = task;
        if (t < p.n_rows) {
            int64_t slot = -1;
            int pos = -1, seq = -1;
            if (t < rows_all) {
                seq = last_not_above(s_row, n, (int)t);
                const int had = s_had[seq];
                if (had & SERVED) {
                    pos = s_start[seq] + (int)t - s_row[seq];
                    const int b = (pos >> bt_shift) - (had & BLOCKS);
                    const int block = b < 0 ? p.a.table[(size_t)seq * p.table_stride + (pos >> bt_shift)] : stack(have - 1 - (s_take[seq] + b));
                    slot = ((int64_t)block << bt_shift) + (pos & (bt - 1));
                }
            }
            p.a.slots[t] = slot, p.a.positions[t] = pos, p.a.row_seq[t] = seq;
            continue;
        }
        t -= p.n_rows;
        if (t < n_parts) {
            const int i = last_not_above(s_part, n + 1, (int)t), np = parts_of(i), local = (int)t - s_part[i];
            const int item = np == 1 ? local : local / np, tile = (int)div_by((uint32_t)item, (uint32_t)p.kv_heads, p.kv_magic);
            const int rows = s_row[i + 1] - s_row[i], tiles = (rows * p.group + p.tile_rows - 1) >> p.tile_shift;
            Kv4Part w;
            w.seq = i < n && (s_had[i] & SERVED) ? i : -1;
            w.row0 = s_row[i];
            w.n_flat = rows * p.group;
            w.start = i < n ? s_start[i] : 0;
            w.tile = tiles - 1 - tile;  // (those that see most come first)
            w.head = item - tile * p.kv_heads;
            w.part_of = (local - item * np) | np << 16;
            w.slot = s_slot[i] + local;
            p.parts[t] = w;
            continue;
        }
        t -= n_parts;
        if (t < taken) {
            const int i = last_not_above(s_take, n, (int)t), b = (s_had[i] & BLOCKS) + (int)t - s_take[i];
            if (b < p.table_stride) p.a.table[(size_t)i * p.table_stride + b] = stack(have - 1 - (int)t);
            continue;
        }
        t -= taken;
        if (left + t < p.n_blocks) p.a.free_blocks[left + t] = stack(left + (int)t);
    }

    if (tid == 0) {
        s_last = arrived == gridDim.x - 1;
        if (s_last && gridDim.x > 1) __hip_atomic_store(p.arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (s_last)
        for (int i = i0; i < i1; ++i) p.a.held_next[i] = s_had[i] & SERVED ? p.end[i] : p.held[i];
}

// ------------------------------------------------------------------------------------------------
// append, read
// ------------------------------------------------------------------------------------------------
template <typename ST>
__device__ __forceinline__ void load8(const ST* p, bool vec, float (&x)[8]) {
    if constexpr (sizeof(ST) == 2) {
        if (vec) {
            const bf16x8 w = *(const bf16x8*)p;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (float)w[e];
            return;
        }
    } else {
        if (vec) {
            const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)p[e];
}

template <int N>
__device__ __forceinline__ void store_words(char* p, const uint32_t (&w)[N]) {
    if constexpr (N == 1) {
        *(uint32_t*)p = w[0];
    } else if constexpr (N == 2) {
        *(u32x2*)p = u32x2{w[0], w[1]};
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) *(u32x4*)(p + 4 * i) = u32x4{w[i], w[i + 1], w[i + 2], w[i + 3]};
    }
}

template <int N>
__device__ __forceinline__ void store_bytes(char* p, const uint32_t (&b)[N]) {
    if constexpr (N == 1) {
        *p = (char)b[0];
    } else if constexpr (N == 2) {
        *(uint16_t*)p = (uint16_t)(b[0] | b[1] << 8);
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) *(uint32_t*)(p + i) = b[i] | b[i + 1] << 8 | b[i + 2] << 16 | b[i + 3] << 24;
    }
}

// tile of a slot's position, and the position in it
template <int HD>
__device__ __forceinline__ char* tile_of(const Kv4Cache& c, int64_t slot, int head, int& key) {
    const int64_t block = slot >> c.block_shift;
    const int in = (int)slot & ((1 << c.block_shift) - 1);
    key = in & 15;
    return c.layer + (((block * c.kv_heads + head) << (c.block_shift - 4)) + (in >> 4)) * (int64_t)Kv4Tile::bytes(HD);
}

// Largest of the four lanes that share a column (lanes i, i + 16, i + 32, i + 48).
__device__ __forceinline__ uint32_t rows4_umax(uint32_t v) {
    const lanes_u32x2 a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(a[0], a[1]);
    const lanes_u32x2 b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(b[0], b[1]);
}

// One wave per 16 rows of one head of K or of V, its lanes as the attention reads a tile: lane (quarter h, row t) has elements
// 8h .. 8h+7 of every group.  Per group: e least with max|x| <= 7 * 2^e, then the nearest level of x / 2^e.  So a group's
// largest magnitude is two lane swaps away, K of 16 rows that fill a tile is written as one run of 1 KB (head_dim 128) and its
// scales as one of 64 bytes; the conversion is the hardware's, which rounds to nearest even and saturates.  Rows that follow
// each other usually lie in one tile, whose lines so come from one workgroup: with the heads of a row together instead, eight
// XCDs wrote parts of each line (79 us where this takes 50: 40 768 rows of 8 heads of 128 in bf16, 211 MB, which a copy moves
// in 41).  Bound by HBM there, by the launch in a decode step (3.8 us).
template <int HD, typename ST>
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4Cache c, int n_rows, const ST* __restrict__ k, int64_t k_row, int64_t k_head,
                                                         const ST* __restrict__ v, int64_t v_row, int64_t v_head, int vec,
                                                         const int64_t* __restrict__ slots, int rows_given, int row0) {
    constexpr int G = HD / 32, LB = HD / 8;
    const int lane = threadIdx.x & 63, h = lane >> 4;
    const uint32_t vecs = blockIdx.x * 4u + (threadIdx.x >> 6);
    const int which = vecs & 1, head = (int)((vecs >> 1) % (uint32_t)c.kv_heads);
    const int64_t row = row0 + (int64_t)((vecs >> 1) / (uint32_t)c.kv_heads) * 16 + (lane & 15);
    const bool there = row < n_rows;
    const int plan_rows = max(c.counts[1] & 0xffffff, rows_given);  // (rows_given: 0 if the slots are the plan's)
    const int64_t slot = there ? slots[row] : -1;
    float x[G][8] = {};
    if (there) {
        const ST* src = (which ? v + row * v_row + head * v_head : k + row * k_row + head * k_head) + h * 8;
#pragma unroll
        for (int g = 0; g < G; ++g) load8(src + g * 32, (vec >> which) & 1, x[g]);
    }
    uint32_t code[G], sc[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[g][e]) & 0x7fffffffu);
        top = rows4_umax(top);
        // the least e with top <= 7 * 2^e = 1.75 * 2^(e+2); biased by 127
        sc[g] = min(max((top >> 23) + ((top & 0x7fffffu) > 0x600000u ? 1u : 0u), SCALE_MIN + 2) - 2, SCALE_MAX);
        const float unit = __uint_as_float(sc[g] << 23);
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[g][0], x[g][1], unit, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[g][2], x[g][3], unit, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[g][4], x[g][5], unit, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[g][6], x[g][7], unit, 3);
        code[g] = w;
        if (top >= 0x7f800000u) sc[g] = SCALE_NAN;
    }
    if (slot < 0 || slot >= c.n_slots || row >= plan_rows) return;  // (the plan's slots behind its rows are those of a plan before)
    int key;
    char* tile = tile_of<HD>(c, slot, head, key);
    if (which == 0) {
        store_words<G>(tile + (h * 16 + key) * LB, code);
        if (h == 0) store_bytes<G>(tile + Kv4Tile::k_scales(HD) + key * G, sc);
    } else {
        constexpr int EPC = HD / 16;  // elements per column
        char* t = tile + Kv4Tile::v_codes(HD) + (key & 3) * (LB / 4) + (key >> 2) * 16 * LB;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            char* at = t + (g * 32 + h * 8) / EPC * LB;
            if constexpr (EPC == 16) *(uint32_t*)(at + (h & 1) * 4) = code[g];
            if constexpr (EPC == 8) *(uint32_t*)at = code[g];
            if constexpr (EPC == 4) {
                *(uint16_t*)at = (uint16_t)code[g];
                *(uint16_t*)(at + LB) = (uint16_t)(code[g] >> 16);
            }
            if constexpr (EPC == 2) {
#pragma unroll
                for (int b = 0; b < 4; ++b) at[b * LB] = (char)(code[g] >> (8 * b));
            }
        }
#pragma unroll
        for (int g = 0; g < G; ++g)
            if (h == (g & 3)) tile[Kv4Tile::v_scales(HD) + g * 16 + key] = (char)sc[g];
    }
}

// Read-back: level times 2^e, exact in fp32 and in bf16.  A thread has 8 elements of a group, whose codes are a word of K or
// lie in one to four columns of V, and writes them as one run; a workgroup has 16 rows of one head of K (of V), then of the
// next, so that each line of the cache is asked for by one XCD.  Bound by HBM: 36.4 us for the 211 MB that a copy moves in 41,
// four fifths of them written.
struct Kv4Work {
    int e8, which, head;
    int64_t row;
};
template <int TPV>
__device__ __forceinline__ Kv4Work work_of(int kv_heads, int row0) {
    const uint64_t idx = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const uint32_t in = (uint32_t)(idx % (16 * TPV)), vec = (uint32_t)(idx / (16 * TPV));
    Kv4Work w;
    w.e8 = in % TPV;
    w.which = vec & 1;
    w.head = (vec >> 1) % (uint32_t)kv_heads;
    w.row = row0 + (int64_t)((vec >> 1) / (uint32_t)kv_heads) * 16 + in / TPV;
    return w;
}

// 8 elements of a word of codes, times their group's scale
__device__ __forceinline__ void values8(uint32_t w, uint32_t sc, bf16x2 (&x)[4]) {
    const float unit = __uint_as_float(sc << 23);
    x[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 0);
    x[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 1);
    x[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 2);
    x[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 3);
}

template <int HD, typename ST>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4Cache c, int n_rows, const int64_t* __restrict__ slots, ST* __restrict__ k,
                                                       ST* __restrict__ v, int row0) {
    constexpr int TPV = HD / 8, LB = HD / 8;
    const Kv4Work w = work_of<TPV>(c.kv_heads, row0);
    const int e8 = w.e8, which = w.which, head = w.head;
    const int64_t row = w.row;
    if (row >= n_rows) return;
    ST* dst = which ? v : k;
    if (!dst) return;
    dst += (row * c.kv_heads + head) * HD + e8 * 8;
    const int64_t slot = slots[row];
    uint32_t code = 0, sc = SCALE_MIN;
    if (slot >= 0 && slot < c.n_slots) {
        int key;
        const char* tile = tile_of<HD>(c, slot, head, key);
        const int g = e8 >> 2;
        if (which == 0) {
            code = *(const uint32_t*)(tile + ((e8 & 3) * 16 + key) * LB + g * 4);
            sc = (uint8_t)tile[Kv4Tile::k_scales(HD) + key * (HD / 32) + g];
        } else {
            constexpr int EPC = HD / 16;
            const char* t = tile + Kv4Tile::v_codes(HD) + (key & 3) * (LB / 4);
            const int col = (key >> 2) * 16 + e8 * 8 / EPC;
            if constexpr (EPC == 16) code = *(const uint32_t*)(t + col * LB + (e8 & 1) * 4);
            if constexpr (EPC == 8) code = *(const uint32_t*)(t + col * LB);
            if constexpr (EPC == 4) code = *(const uint16_t*)(t + col * LB) | (uint32_t) * (const uint16_t*)(t + (col + 1) * LB) << 16;
            if constexpr (EPC == 2) {
#pragma unroll
                for (int b = 0; b < 4; ++b) code |= (uint32_t)(uint8_t)t[(col + b) * LB] << (8 * b);
            }
            sc = (uint8_t)tile[Kv4Tile::v_scales(HD) + g * 16 + key];
        }
    }
    bf16x2 x[4];
    values8(code, sc, x);
    if (sc == SCALE_NAN) {
        const bf16x2 nan = {(__bf16)__builtin_nanf(""), (__bf16)__builtin_nanf("")};
#pragma unroll
        for (int b = 0; b < 4; ++b) x[b] = nan;
    }
    if constexpr (sizeof(ST) == 2) {
        bf16x8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = x[e >> 1][e & 1];
        *(bf16x8*)dst = o;
    } else {
        f32x4 a, b;
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] = (float)x[e >> 1][e & 1], b[e] = (float)x[2 + (e >> 1)][e & 1];
        *(f32x4*)dst = a;
        *(f32x4*)(dst + 4) = b;
    }
}

// ------------------------------------------------------------------------------------------------
// attention
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ bf16x8 frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    const u32x4 w = {a, b, c, d};
    return __builtin_bit_cast(bf16x8, w);
}

template <int B>  // byte B of the words, as two bf16 in a word, times the scale
__device__ __forceinline__ uint32_t pair_of(uint32_t w, float unit) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, B));
}

__device__ __forceinline__ uint32_t pair_of(uint32_t w, float unit, int b) {
    switch (b) {
        case 0: return pair_of<0>(w, unit);
        case 1: return pair_of<1>(w, unit);
        case 2: return pair_of<2>(w, unit);
        default: return pair_of<3>(w, unit);
    }
}

template <int HD>
struct KeyRegs {  // of one tile of 16 positions
    uint32_t w[HD / 32];
    uint32_t sc[HD / 128 > 1 ? HD / 128 : 1];  // scales of the lane's key
};
template <int HD>
struct ValueRegs {
    uint32_t w[HD / 32];
    uint32_t sc;  // of the lane's four keys, in its column's group
};

// The pool, as an address that the compiler knows to be global memory (a flat load would also wait for LDS).  An unsigned offset
// from an address that all lanes share costs no arithmetic.
#define EE_GLOBAL __attribute__((address_space(1)))
typedef const EE_GLOBAL char* PoolPtr;

// PAST: without keeping the lines in the caches.
template <bool PAST, int N>
__device__ __forceinline__ void load_words(PoolPtr p, uint32_t (&w)[N]) {
    if constexpr (N == 1) {
        w[0] = *(const EE_GLOBAL uint32_t*)p;
    } else if constexpr (N == 2) {
        const u32x2 x = PAST ? __builtin_nontemporal_load((const EE_GLOBAL u32x2*)p) : *(const EE_GLOBAL u32x2*)p;
        w[0] = x[0], w[1] = x[1];
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const u32x4 x = PAST ? __builtin_nontemporal_load((const EE_GLOBAL u32x4*)(p + 4 * i)) : *(const EE_GLOBAL u32x4*)(p + 4 * i);
            w[i] = x[0], w[i + 1] = x[1], w[i + 2] = x[2], w[i + 3] = x[3];
        }
    }
}

template <int HD, bool PAST>
__device__ __forceinline__ void load_keys(PoolPtr tile, uint32_t lane, KeyRegs<HD>& r) {
    constexpr uint32_t LB = HD / 8, G = HD / 32;
    load_words<PAST, G>(tile + lane * LB, r.w);
    PoolPtr sc = tile + Kv4Tile::k_scales(HD) + (lane & 15u) * G;
    if constexpr (G == 1) r.sc[0] = *(const EE_GLOBAL uint8_t*)sc;
    if constexpr (G == 2) r.sc[0] = *(const EE_GLOBAL uint16_t*)sc;
    if constexpr (G >= 4) load_words<false, G / 4>(sc, r.sc);
}
template <int HD, bool PAST>
__device__ __forceinline__ void load_values(PoolPtr tile, uint32_t lane, ValueRegs<HD>& r) {
    constexpr uint32_t LB = HD / 8, G = HD / 32;
    load_words<PAST, G>(tile + Kv4Tile::v_codes(HD) + lane * LB, r.w);
    r.sc = *(const EE_GLOBAL uint32_t*)(tile + Kv4Tile::v_scales(HD) + ((lane & 15u) * HD / 512u * 16u + (lane >> 4) * 4u));
}

__device__ __forceinline__ float scale_of(uint32_t word, int i) {  // byte i as 2^(byte - 127)
    return __uint_as_float((word >> (8 * i) & 255u) << 23);
}

__device__ __forceinline__ uint32_t bytes_255(uint32_t w) {  // 0x80 in every byte of w that is 255 (and maybe above such a one)
    const uint32_t x = ~w;
    return (x - 0x01010101u) & ~x & 0x80808080u;
}

// What one workgroup leaves for another one of the same launch, maybe on another XCD.
__device__ __forceinline__ void hand_over2(float* p, f32x2 v) {
    __hip_atomic_store((uint64_t*)p, __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 handed2(const float* p) {
    return __builtin_bit_cast(f32x2, __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
__device__ __forceinline__ void hand_over1(float* p, float v) {
    __hip_atomic_store((uint32_t*)p, __float_as_uint(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float handed1(const float* p) {
    return __uint_as_float(__hip_atomic_load((const uint32_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// l + both of a pair of bf16, in one instruction (fp32, within one unit in the last place of the sum)
__device__ __forceinline__ float add_pair(uint32_t pair, float l) {
    const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), one, l, false);
}

// parts that are joined at a time: all, or of many about their number's square root
__device__ __forceinline__ int fan_shift_of(int n_parts) { return n_parts <= 16 ? 4 : n_parts <= 64 ? 3 : n_parts <= 256 ? 4 : 5; }

// The workgroup has a part, of a plan that the launch was made for: else nobody writes, so that no array is left and no counter of
// parts stays behind.
__device__ __forceinline__ bool of_this_plan(const Kv4Attend& a) {
    const u32x2 counts = *(const u32x2*)a.counts;  // (in one load, beside that of the part)
    return (blockIdx.x < counts[0]) & (counts[0] <= (uint32_t)a.grid) & (counts[1] == (uint32_t)a.shape);
}

// row of an entry in its request; where the entry's results go
__device__ __forceinline__ int row_of(const Kv4Attend& a, int f) { return (int)div_by((uint32_t)f, (uint32_t)a.group, a.group_magic); }
__device__ __forceinline__ size_t out_row(const Kv4Attend& a, const Kv4Part& w, int f) {
    const int row = row_of(a, f);
    return (size_t)(w.row0 + row) * (a.group * a.kv_heads) + w.head * a.group + f - row * a.group;
}

// chunks first .. end of part `part` of `n_parts` that n_chunks from c_first on are cut into, as evenly as they can be
__device__ __forceinline__ void part_of_chunks(int c_first, int n_chunks, int n_parts, int part, int& first, int& end) {
    const int each = div_small(n_chunks, n_parts), more = n_chunks - each * n_parts;
    first = c_first + part * each + min(part, more);
    end = first + each + (part < more ? 1 : 0);
}

// rows that see nothing
template <int HD, typename ST>
__device__ __forceinline__ void sees_nothing(const Kv4Attend& a, const Kv4Part& w, int f0, int f_end, int threads, ST* out) {
    for (int i = threadIdx.x; i < (f_end - f0) * HD; i += threads) {
        const int f = f0 + i / HD;
        const size_t o = out_row(a, w, f);
        out[o * HD + i % HD] = (ST)0.f;
        if (i % HD == 0 && a.lse) a.lse[o] = -INFINITY;
    }
}

__device__ __forceinline__ void store_pair(float* p, f32x2 x) { *(f32x2*)p = x; }
__device__ __forceinline__ void store_pair(__bf16* p, f32x2 x) { *(bf16x2*)p = __builtin_convertvector(x, bf16x2); }

// What a thread has in a pass over a part's M rows: pairs of elements of one row, and where a part holds them.  Each store or load
// of a wave is of whole lines, as what goes past the caches is not put together there.
template <int HD, int THREADS, int M>
struct PartPlace {
    // rows one after the other, a thread's pairs LANES apart
    static constexpr int PAIRS = M * HD / 2 >= 4 * THREADS ? 4 : M * HD / 2 >= 2 * THREADS ? 2 : 1, LANES = HD / 2 / PAIRS;
    static constexpr int ROWS = THREADS / LANES, PASSES = (M + ROWS - 1) / ROWS;
    int row, at;
    __device__ __forceinline__ explicit PartPlace(int pass) : row(pass * ROWS + threadIdx.x / LANES), at(threadIdx.x % LANES * 2) {}
    __device__ __forceinline__ bool first() const { return at == 0; }
    __device__ __forceinline__ int element(int i) const { return at + 2 * LANES * i; }
    __device__ __forceinline__ int held(int i) const { return row * HD + element(i); }
};
template <int HD>
struct PartPlace<HD, 512, KV4_WIDE> {
    // as the registers of the prompts' kernel hold them: [32 rows each of a wave][column of V within its half][pair][lane]
    static constexpr int PAIRS = HD / 32, PASSES = 4;
    int row, column, at;
    __device__ __forceinline__ PartPlace(int wave, int i) {  // i: 8 of a lane's columns
        const int lane = threadIdx.x & 63;
        row = 32 * wave + (lane & 31);
        column = 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
        at = ((wave * 8 + i) * PAIRS * 64 + lane) * 2;
    }
    __device__ __forceinline__ explicit PartPlace(int pass) : PartPlace((threadIdx.x >> 6) & 3, (threadIdx.x >> 8) * 4 + pass) {}
    __device__ __forceinline__ bool first() const { return column == 0; }
    __device__ __forceinline__ int element(int b) const { return column * (HD / 16) + 2 * b; }
    __device__ __forceinline__ int held(int b) const { return at + b * 128; }
};

// Parts are joined by the workgroup that leaves the last one, in their order; many of them in two levels: first each FAN_IN
// neighbours by the last of those, into the first one's place, then these.  The parts go past the caches of this XCD (agent-scope
// stores and loads).  Fences instead act on the whole of its L2: a release cost a launch of 1024 parts 300 us, and an acquire
// by the workgroups that join alone made a ragged batch's 20 us 37.
// APART: the log-sum-exp's sums come apart from the results' (see below).
template <int HD, int THREADS, int M, bool APART, typename ST>
__device__ __forceinline__ void join_parts(const Kv4Attend& a, const Kv4Part& w, int n_parts, int f0, int f_end, uint32_t* s_last) {
    const int part = w.part_of & 0xffff, slot0 = w.slot - part;
    const int fan_shift = fan_shift_of(n_parts), fan = 1 << fan_shift;
    const int groups = (n_parts + fan - 1) >> fan_shift, group0 = part >> fan_shift << fan_shift;
    ST* out = (ST*)a.out;
    const bool two_levels = groups > 1;
    int first = slot0 + group0, stride = 1, n = min(fan, n_parts - group0);
    uint32_t* counter = a.arrived + first;
    const float *part_ml = a.part_ml, *part_l = a.part_l;
    for (int level = 0;; ++level) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // each thread's stores have arrived before its workgroup is counted
        __syncthreads();
        if (threadIdx.x == 0) {
            const uint32_t before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if ((int)before == n - 1) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            *s_last = before;
        }
        __syncthreads();
        if ((int)*s_last != n - 1) return;
        const bool whole = level == 1 || !two_levels;
        // a thread has PAIRS pairs of elements of a row and asks for all of them of up to eight parts at once
        using Place = PartPlace<HD, THREADS, M>;
        constexpr int PAIRS = Place::PAIRS;
        for (int pass = 0; pass < Place::PASSES; ++pass) {
            const Place here(pass);
            const int r = here.row;
            if (r >= f_end - f0) continue;
            const size_t row = (size_t)first * M + r, step = (size_t)stride * M;
            const float* o = a.part_o + (size_t)first * (M * HD);
            float top = -INFINITY, sum = 0.f, sum_lse = 0.f;
            f32x2 acc[PAIRS] = {};
            auto add = [&](auto at_once, int v0) {
                constexpr int N = decltype(at_once)::value;
                f32x2 ml[N], x[N][PAIRS];
                float lse[APART ? N : 1];
#pragma unroll
                for (int v = 0; v < N; ++v) {
                    const size_t at = step * min(v0 + v, n - 1);  // (no branch, so that no load waits for another one)
                    ml[v] = handed2(part_ml + 2 * (row + at));
                    if constexpr (APART) lse[v] = handed1(part_l + row + at);
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) x[v][i] = handed2(o + at * HD + here.held(i));
                }
                float t = top;
#pragma unroll
                for (int v = 0; v < N; ++v) t = fmaxf(t, ml[v][0]);
                const float ref = t == -INFINITY ? 0.f : t;
                const float old = __builtin_amdgcn_exp2f(top - ref);
                sum *= old;
                if constexpr (APART) sum_lse *= old;
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) acc[i] *= old;
#pragma unroll
                for (int v = 0; v < N; ++v) {
                    if (v0 + v >= n) break;
                    const float wt = __builtin_amdgcn_exp2f(ml[v][0] - ref);
                    sum += wt * ml[v][1];
                    if constexpr (APART) sum_lse += wt * lse[v];
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) acc[i] += wt * x[v][i];
                }
                top = t;
            };
            for (int v0 = 0; v0 < n; v0 += 8) {
                if (n - v0 <= 2)
                    add(std::integral_constant<int, 2>(), v0);
                else
                    add(std::integral_constant<int, 8>(), v0);
            }
            const int f = f0 + r;
            if (whole) {
                const size_t at = out_row(a, w, f);
                const float inv = 1.f / sum;
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) store_pair(out + at * HD + here.element(i), acc[i] * inv);
                if (a.lse && here.first()) a.lse[at] = ((top == -INFINITY ? 0.f : top) + log2f(APART ? sum_lse : sum)) * 0.6931471805599453f;
            } else {
                // elements into the first part's place, which no other thread reads; weights apart, as all of a row's threads
                // read them
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) hand_over2((float*)o + here.held(i), acc[i]);
                if (here.first()) {
                    hand_over2(a.joined_ml + 2 * row, f32x2{top, sum});
                    if constexpr (APART) hand_over1(a.joined_l + row, sum_lse);
                }
            }
        }
        if (whole) return;
        counter = a.arrived_groups + slot0;
        part_ml = a.joined_ml, part_l = a.joined_l;
        first = slot0, stride = fan, n = groups;
    }
}

// Attention of one part: up to 16 * UNITS entries (row, query head) of a kv head over a run of chunks of 32 positions, by NW waves
// that take every NW-th chunk.  With s = scale * q.k in units of ln 2, running maximum m and weights 2^(s - m):
//   l <- l 2^(m - m') + sum 2^(s - m'),   o <- o 2^(m - m') + sum 2^(s - m') v,   m' = max(m, s),   out = o / l.
// o and l are rescaled only when some maximum has grown by more than a factor 2^8 of the weights, which leaves them in fp32's
// range; m, l and o are fp32.  Shares are joined in the same way: waves through LDS, parts through join_parts.  A row that gets
// there sees its own position at least, so l is at least 1, unless all of its scores are -inf: then 0 / 0 is the NaN that the
// formula gives.
// Products are 16x16x32 bf16 with positions as rows of the first (S^T = K Q^T): its result then lies in the lanes that the second one
// (O^T = V^T P^T) wants its probabilities in, if V's tile has its positions in that order, and nothing moves between lanes.  K and
// V are exact in bf16.  NT: bf16 terms of an element of Q (1: Q is bf16; 3: fp32, exactly), PT: of a probability: three for the
// fp32 model, two for the tiles of 16, which wait for memory anyway (error against 64 bits 0.0017, all of it the result's own
// rounding to bf16), one for larger ones (0.0021; a second term costs them a sixth of their time: 64 requests of 500
// to 16 384 positions and 5 rows, 32 heads on 8, 171 us instead of 144).  With one term the divisor is the sum of the rounded
// probabilities: the weights that V gets add to one, so a row in which one position outweighs the others keeps that one's value,
// whatever its weight rounds to.  The log-sum-exp, where it is asked for (LSE), has a sum of its own, of the probabilities before
// they are rounded (those 64 requests 151 us).  UNITS: 16 entries each of a tile.
// Bound by HBM where contexts are long: 64 requests of up to 16 384 positions, 32 heads on 8 of 128 elements, 589 MB: 114 us,
// 5.2 TB/s (a copy's rate is 5.15), every byte read once.  So what counts is what is on its way: of the tiles DEPTH steps ahead
// each load is asked for as soon as its registers have been read.  One request of 131 071 positions: 32 us for 143 MB, 4.5
// TB/s; of which 4 us are its parts' joins.  16 requests of up to 2048 positions, 32 heads: 19 us for 69 MB, launch and last
// parts included.  A single user's 513 positions (6.7 us) are bound by the launch and the chain part, table, K, V, join.
template <int HD, int NT, int PT, int UNITS, int NW, int DEPTH, bool PAST, bool LSE, typename ST>
__global__ __launch_bounds__(NW * 64, HD > 128 ? 1 : UNITS > 1 || DEPTH > 1 ? 2 : NT == 1 ? 4 : 3) void kv4_attend_kernel(Kv4Attend a) {
    constexpr int G = HD / 32, EPC = HD / 16, M = 16 * UNITS;
    constexpr int CT = KV4_CHUNK / 16;  // tiles of 16 positions at a time: one contraction of P.V
    static_assert(CT == 2, "a contraction has 32 positions");
    constexpr int LDO = HD + 4;
    constexpr bool APART = LSE && PT == 1;
    __shared__ float s_o[NW * 16 * LDO];
    __shared__ float s_m[NW * 16], s_l[NW * 16], s_lse[APART ? NW * 16 : 1];
    __shared__ uint32_t s_last;

    const Kv4Part w = a.parts[blockIdx.x];  // (there is room for as many as the grid has; asked for together with their number)
    if (!of_this_plan(a)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const int f0 = w.tile * M, f_end = min(w.n_flat, f0 + M);  // entries
    ST* out = (ST*)a.out;
    if (w.seq < 0) {
        sees_nothing<HD>(a, w, f0, f_end, NW * 64, out);
        return;
    }

    // entry f0 + 16 u + col of this lane: row, position, first and last position it sees
    bf16x8 q[UNITS][NT][G];
    int lo[UNITS], hi[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const int f = min(f0 + 16 * u + col, f_end - 1);  // (columns behind the last entry repeat it; nobody reads them)
        const int row = row_of(a, f), head = w.head * a.group + f - row * a.group;
        hi[u] = w.start + row;
        lo[u] = a.window ? max(0, hi[u] - a.window + 1) : 0;
        const ST* src = (const ST*)a.q + (w.row0 + row) * a.q_row + head * a.q_head + quarter * 8;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if constexpr (sizeof(ST) == 2) {
                if (a.q_vec) {
                    q[u][0][g] = *(const bf16x8*)(src + g * 32);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) q[u][0][g][e] = src[g * 32 + e];
                }
            } else {
                float x[8];
                load8(src + g * 32, a.q_vec, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float rest = x[e];
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        q[u][t][g][e] = (__bf16)rest;
                        rest -= (float)q[u][t][g][e];
                    }
                }
            }
        }
    }
    const int pos_first = w.start + row_of(a, f0), pos_last = w.start + row_of(a, f_end - 1);
    const int lo_min = a.window ? max(0, pos_first - a.window + 1) : 0;
    const int lo_max = a.window ? max(0, pos_last - a.window + 1) : 0;
    const int c_first = lo_min / KV4_CHUNK, n_chunks = pos_last / KV4_CHUNK + 1 - c_first;
    // (a tile that sees less than the request's last row, because of its rows' positions or the window, needs fewer parts)
    const int n_parts = min(w.part_of >> 16, max(1, div_small(n_chunks + a.min_chunks - 1, a.min_chunks))), part = w.part_of & 0xffff;
    if (part >= n_parts) return;
    int c_lo, c_hi;
    part_of_chunks(c_first, n_chunks, n_parts, part, c_lo, c_hi);

    const int32_t* table = a.table + (size_t)w.seq * a.table_stride;
    const int last_tile = pos_last >> 4;
    const size_t block_bytes = ((size_t)Kv4Tile::bytes(HD) << a.tiles_shift) * a.kv_heads;
    const PoolPtr base = (PoolPtr)a.layer + ((size_t)Kv4Tile::bytes(HD) << a.tiles_shift) * w.head;
    const int in_block = (1 << a.tiles_shift) - 1;

    // step `it` of this wave: chunk c_lo + wave + it * NW, two tiles; a tile behind the last one that is seen repeats it (its
    // positions are hidden)
    const int n_it = max(0, (c_hi - c_lo - wave + NW - 1) / NW);
    auto tile_at = [&](int it, int t) { return (c_lo + wave + it * NW) * CT + t; };
    // block numbers of AHEAD steps at a time, one per lane, and those of the next
    constexpr int AHEAD = 64 / CT;
    auto blocks_from = [&](int it) {
        const int t = min(tile_at(it + lane / CT, lane % CT), last_tile);
        return table[t >> a.tiles_shift];
    };
    int blocks = n_it ? blocks_from(0) : 0, blocks_next = n_it > AHEAD ? blocks_from(AHEAD) : 0;
    auto tile_addr = [&](int it, int t) {
        const int tile = min(tile_at(it, t), last_tile);
        const int block = __builtin_amdgcn_readlane(blocks, it % AHEAD * CT + t);
        return base + (size_t)block * block_bytes + (size_t)(tile & in_block) * Kv4Tile::bytes(HD);
    };

    f32x4 o[UNITS][EPC];
    // m: the scores' reference, at most a.slack below their maximum (so no probability passes 2^8)
    float m[UNITS], l[UNITS], l_lse[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        m[u] = -INFINITY, l[u] = l_lse[u] = 0.f;
#pragma unroll
        for (int j = 0; j < EPC; ++j) o[u][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // K of a step DEPTH ahead is asked for as soon as K of this one has been used, V likewise
    KeyRegs<HD> key_regs[DEPTH][CT];
    ValueRegs<HD> value_regs[DEPTH][CT];
    PoolPtr at[CT];
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
        if (i < n_it) {
#pragma unroll
            for (int t = 0; t < CT; ++t) at[t] = tile_addr(i, t);
#pragma unroll
            for (int t = 0; t < CT; ++t) load_keys<HD, PAST>(at[t], lane, key_regs[i][t]);
#pragma unroll
            for (int t = 0; t < CT; ++t) load_values<HD, PAST>(at[t], lane, value_regs[i][t]);
        }
    }
    auto step = [&](const int it, KeyRegs<HD>(&kr)[CT], ValueRegs<HD>(&vr)[CT]) {
        const int key0 = tile_at(it, 0) * 16;
        // scores: rows = positions, columns = entries
        f32x4 s[UNITS][CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) {
#pragma unroll
            for (int u = 0; u < UNITS; ++u) s[u][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float unit = scale_of(kr[t].sc[g >> 2], g & 3);
                const bf16x8 kf = frag(pair_of<0>(kr[t].w[g], unit), pair_of<1>(kr[t].w[g], unit), pair_of<2>(kr[t].w[g], unit),
                                       pair_of<3>(kr[t].w[g], unit));
#pragma unroll
                for (int u = 0; u < UNITS; ++u)
#pragma unroll
                    for (int n = NT - 1; n >= 0; --n) s[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[u][n][g], s[u][t], 0, 0, 0);
            }
        }
        const bool more = it + DEPTH < n_it;
        if (more) {
            if ((it + DEPTH) % AHEAD == 0) {
                blocks = blocks_next;
                blocks_next = blocks_from(it + DEPTH + AHEAD);
            }
#pragma unroll
            for (int t = 0; t < CT; ++t) at[t] = tile_addr(it + DEPTH, t);
#pragma unroll
            for (int t = 0; t < CT; ++t) load_keys<HD, PAST>(at[t], lane, kr[t]);
        }
        bool poisoned = false;
        uint32_t nan_keys[CT] = {};  // bytes 1 where V of the lane's key and group is NaN
        if (key0 + 16 * CT > pos_first + 1 || key0 < lo_max) {  // some entry does not see all of these positions
            int key_lane = key0 + quarter * 4;  // position of s[u][t][i]: key_lane + 16 t + i
            asm volatile("" : "+v"(key_lane));  // (nothing of this branch is worth computing outside of it)
            bool any = false;
#pragma unroll
            for (int t = 0; t < CT; ++t) {
#pragma unroll
                for (int u = 0; u < UNITS; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = key_lane + 16 * t + i;
                        if (key > hi[u] || key < lo[u]) s[u][t][i] = -INFINITY;
                    }
                // V behind the last position that any entry sees may hold anything: a scale of 1 makes it finite, and its
                // probabilities are zero
                uint32_t keep = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (key_lane + 16 * t + i <= pos_last) keep |= 255u << (8 * i);
                vr[t].sc = (vr[t].sc & keep) | (0x7f7f7f7fu & ~keep);
                any |= bytes_255(vr[t].sc) != 0;
            }
            poisoned = __any(any);
            if (poisoned) {  // NaN in V that not every entry sees: taken out here, put back below
#pragma unroll
                for (int t = 0; t < CT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if ((vr[t].sc >> (8 * i) & 255u) == SCALE_NAN) vr[t].sc ^= 128u << (8 * i), nan_keys[t] |= 1u << (8 * i);
            }
        }
        u32x4 pf[UNITS][PT];
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            float top = s[u][0][0];
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, s[u][t][i]);
            top = fmaxf(rows4_max(top), m[u]);
            if (__any(top > m[u] + a.slack)) {
                const float corr = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[u] - top) * a.scale_log2);
                l[u] *= corr;
                if constexpr (APART) l_lse[u] *= corr;
#pragma unroll
                for (int j = 0; j < EPC; ++j) o[u][j] *= corr;
                m[u] = top;
            }
            const float ref = m[u] == -INFINITY ? 0.f : m[u] * a.scale_log2;
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    f32x2 p;
                    p[0] = __builtin_amdgcn_exp2f(fmaf(s[u][t][i], a.scale_log2, -ref));
                    p[1] = __builtin_amdgcn_exp2f(fmaf(s[u][t][i + 1], a.scale_log2, -ref));
                    if constexpr (PT > 1) l[u] += p[0] + p[1];
                    if constexpr (APART) l_lse[u] += p[0] + p[1];
#pragma unroll
                    for (int n = 0; n < PT; ++n) {
                        const uint32_t h = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
                        if constexpr (PT == 1) l[u] = add_pair(h, l[u]);
                        pf[u][n][t * 2 + (i >> 1)] = h;
                        if (n + 1 < PT) p[0] -= __uint_as_float(h << 16), p[1] -= __uint_as_float(h & 0xffff0000u);
                    }
                }
        }
        // weighted sum: rows = elements (column c of V's layout), columns = entries
        float u0[4], u1[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u0[i] = scale_of(vr[0].sc, i), u1[i] = scale_of(vr[1].sc, i);
#pragma unroll
        for (int b = 0; b < EPC / 2; ++b) {
            uint32_t x0[4], x1[4];  // elements 2b, 2b+1 of the column, at the four keys
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int byte = i * (HD / 32) + b;  // of the lane's codes
                x0[i] = pair_of(vr[0].w[byte >> 2], u0[i], byte & 3);
                x1[i] = pair_of(vr[1].w[byte >> 2], u1[i], byte & 3);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t sel = h ? 0x07060302u : 0x05040100u;
                const bf16x8 vf = frag(__builtin_amdgcn_perm(x0[1], x0[0], sel), __builtin_amdgcn_perm(x0[3], x0[2], sel),
                                       __builtin_amdgcn_perm(x1[1], x1[0], sel), __builtin_amdgcn_perm(x1[3], x1[2], sel));
#pragma unroll
                for (int u = 0; u < UNITS; ++u)
#pragma unroll
                    for (int n = PT - 1; n >= 0; --n)
                        o[u][2 * b + h] =
                            __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, pf[u][n]), o[u][2 * b + h], 0, 0, 0);
            }
        }
        if (more) {
#pragma unroll
            for (int t = 0; t < CT; ++t) load_values<HD, PAST>(at[t], lane, vr[t]);
        }
        if (poisoned) {
            // an entry that sees a position whose group of V is NaN gets NaN there, one that does not sees zero: the product of
            // "is NaN" and "is seen", both 0 or 1, counts them
            int key_lane = key0 + quarter * 4;
            asm volatile("" : "+v"(key_lane));
            bf16x8 is_nan;
#pragma unroll
            for (int e = 0; e < 8; ++e) is_nan[e] = (__bf16)(float)(nan_keys[e >> 2] >> (8 * (e & 3)) & 1u);
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                bf16x8 seen;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int key = key_lane + 16 * (e >> 2) + (e & 3);
                    seen[e] = (__bf16)(key <= hi[u] && key >= lo[u] ? 1.f : 0.f);
                }
                const f32x4 count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(is_nan, seen, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int j = 0; j < EPC; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (count[i] > 0.f) o[u][j][i] = __builtin_nanf("");
            }
        }
    };
    for (int it = 0; it < n_it; it += DEPTH) {
#pragma unroll
        for (int i = 0; i < DEPTH; ++i)
            if (i == 0 || it + i < n_it) step(it + i, key_regs[i], value_regs[i]);
    }

    // join the waves' shares, 16 entries at a time
    constexpr int EPT = 16 * HD >= 2 * NW * 64 ? 16 * HD / (NW * 64) : 2;  // elements per thread
    constexpr int TPR = HD / EPT;  // threads of a row, whose pairs of elements lie next to each other
    const int my_row = threadIdx.x / TPR, my_d = threadIdx.x % TPR * 2;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        if (f0 + 16 * u >= f_end) break;
        const float lsum = rows4_sum(l[u]), lse_sum = APART ? rows4_sum(l_lse[u]) : 0.f;
        if (u) __syncthreads();
        if (f0 + 16 * u + col < f_end) {
            float* dst = s_o + (wave * 16 + col) * LDO;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < EPC; ++j) dst[(quarter * 4 + i) * EPC + j] = o[u][j][i];
            if (quarter == 0) {
                s_m[wave * 16 + col] = m[u] * a.scale_log2, s_l[wave * 16 + col] = lsum;
                if constexpr (APART) s_lse[wave * 16 + col] = lse_sum;
            }
        }
        __syncthreads();
        const int f = f0 + 16 * u + my_row;
        if (my_row < 16 && f < f_end) {
            float top = -INFINITY, sum = 0.f, sum_lse = 0.f, acc[EPT];
#pragma unroll
            for (int v = 0; v < NW; ++v) top = fmaxf(top, s_m[v * 16 + my_row]);
            const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int e = 0; e < EPT; ++e) acc[e] = 0.f;
#pragma unroll
            for (int v = 0; v < NW; ++v) {
                const float wt = __builtin_amdgcn_exp2f(s_m[v * 16 + my_row] - ref);
                sum += wt * s_l[v * 16 + my_row];
                if constexpr (APART) sum_lse += wt * s_lse[v * 16 + my_row];
                // (a wave that saw nothing has weight zero and zeros)
#pragma unroll
                for (int e = 0; e < EPT; ++e) acc[e] += wt * s_o[(v * 16 + my_row) * LDO + my_d + (e >> 1) * (2 * TPR) + (e & 1)];
            }
            if (n_parts == 1) {
                const size_t r = out_row(a, w, f);
                const float inv = 1.f / sum;
#pragma unroll
                for (int e = 0; e < EPT; e += 2) store_pair(out + r * HD + my_d + e * TPR, f32x2{acc[e] * inv, acc[e + 1] * inv});
                if (a.lse && my_d == 0) a.lse[r] = (ref + log2f(APART ? sum_lse : sum)) * 0.6931471805599453f;
            } else {
                const size_t r = (size_t)w.slot * M + 16 * u + my_row;
#pragma unroll
                for (int e = 0; e < EPT; e += 2) hand_over2(a.part_o + r * HD + my_d + e * TPR, f32x2{acc[e], acc[e + 1]});
                if (my_d == 0) {
                    hand_over2(a.part_ml + 2 * r, f32x2{top, sum});
                    if constexpr (APART) hand_over1(a.part_l + r, sum_lse);
                }
            }
        }
    }
    if (n_parts > 1) join_parts<HD, NW * 64, M, APART, ST>(a, w, n_parts, f0, f_end, &s_last);
}

// Prompts: 128 entries of a tile, 32 for each of four waves.  The four convert the next 32 positions together, a tile of K or V
// each, into bf16 in LDS in operand order, while they work on these; so an element is converted once for 128 entries, and
// 32 x 32 products halve what is read from LDS per operation.  One barrier per 32 positions, two buffers.  Two such groups of
// waves take every other 32 positions, so that a SIMD has two waves, and join their sums through LDS at the end.
// One bf16 term of a probability, divided by the sum of the rounded ones as above (error against 64 bits 0.0023, of which the
// result's rounding is 0.0017; a second term would be half as many products again).
// 1024 rows at the end of 8192 positions, 32 heads on 8 of 128 elements, 129 GFLOP: 146 us, 885 TFLOP/s, where a large matrix
// product reaches 1215.  The vector units' work (per score an exponential, a multiply-add, a maximum, half a sum and conversion)
// takes about as long as the products, and two waves of a SIMD overlap them in part; LDS is active a third of the time.  Three
// groups of waves with Q in LDS: 151 us.
template <bool LSE>
__global__ __launch_bounds__(512, 2) void kv4_attend_wide_kernel(Kv4Attend a) {
    constexpr int HD = 128, M = KV4_WIDE, G = HD / 32, EPC = HD / 16, KS = HD / 16, DB = HD / 32, LB = HD / 8;
    __shared__ u32x4 s_operands[2][2][(KS + 2 * DB) * 64];  // K, V of each group's two steps; at the end the second group's sums
    __shared__ float s_ml[LSE ? 3 : 2][256];
    __shared__ uint32_t s_scales_of[2][2][2][G * 4];  // of V, if some entry does not see all of the positions
    __shared__ uint32_t s_nan_of[2][2][2];            // ... and there is a NaN among them
    static_assert(sizeof(s_operands) >= 4 * 64 * 16 * DB * sizeof(float), "room for the sums");
    __shared__ uint32_t s_last;

    const Kv4Part w = a.parts[blockIdx.x];
    if (!of_this_plan(a)) return;
    const int lane = threadIdx.x & 63, group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 3;
    const int col = lane & 31, half = lane >> 5;
    const int f0 = w.tile * M, f_end = min(w.n_flat, f0 + M);
    __bf16* out = (__bf16*)a.out;
    if (w.seq < 0) {
        sees_nothing<HD>(a, w, f0, f_end, 512, out);
        return;
    }

    // entry of this lane's column; what the wave's and the workgroup's entries see
    const int f_wave = f0 + 32 * wave, f = min(f_wave + col, f_end - 1);
    const int row = row_of(a, f), head = w.head * a.group + f - row * a.group;
    const int hi = w.start + row, lo = a.window ? max(0, hi - a.window + 1) : 0;
    bf16x8 q[KS];  // elements 16 s + 8 half ..
    {
        const __bf16* src = (const __bf16*)a.q + (w.row0 + row) * a.q_row + head * a.q_head + half * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if (a.q_vec) {
                q[s] = *(const bf16x8*)(src + s * 16);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) q[s][e] = src[s * 16 + e];
            }
        }
    }
    auto first_of = [&](int pos) { return a.window ? max(0, pos - a.window + 1) : 0; };
    const int pos_first = w.start + row_of(a, f0), pos_last = w.start + row_of(a, f_end - 1);
    const bool idle = f_wave >= f_end;
    const int wave_first = w.start + row_of(a, min(f_wave, f_end - 1)), wave_last = w.start + row_of(a, min(f_wave + 31, f_end - 1));
    const int c_first = first_of(pos_first) / KV4_CHUNK, n_chunks = pos_last / KV4_CHUNK + 1 - c_first;
    // (a tile that sees less than the request's last row, because of its rows' positions or the window, needs fewer parts)
    const int n_parts = min(w.part_of >> 16, max(1, div_small(n_chunks + a.min_chunks - 1, a.min_chunks))), part = w.part_of & 0xffff;
    if (part >= n_parts) return;
    int c_lo, c_hi;
    part_of_chunks(c_first, n_chunks, n_parts, part, c_lo, c_hi);

    // this wave converts tile `tl` of a step's two, of K or of V
    const int tl = wave & 1, quarter = lane >> 4, t16 = lane & 15;
    const bool of_v = wave >= 2;
    const int32_t* table = a.table + (size_t)w.seq * a.table_stride;
    const int last_tile = pos_last >> 4, in_block = (1 << a.tiles_shift) - 1;
    const size_t block_bytes = ((size_t)Kv4Tile::bytes(HD) << a.tiles_shift) * a.kv_heads;
    const PoolPtr base = (PoolPtr)a.layer + ((size_t)Kv4Tile::bytes(HD) << a.tiles_shift) * w.head;
    auto(&s_buffers)[2][(KS + 2 * DB) * 64] = s_operands[group];
    auto(&s_scales)[2][2][G * 4] = s_scales_of[group];
    auto(&s_nan)[2][2] = s_nan_of[group];
    const int n_it = max(0, (c_hi - c_lo - group + 1) >> 1), n_most = (c_hi - c_lo + 1) >> 1;
    auto chunk_of = [&](int it) { return c_lo + group + 2 * it; };
    // where the tiles of 64 steps lie, one per lane, and the block numbers of the 64 behind them
    auto tile_of_lane = [&](int it) { return min(chunk_of(it + lane) * 2 + tl, last_tile); };
    auto offsets_of = [&](int it, int block) { return (uint64_t)block * block_bytes + (uint32_t)((tile_of_lane(it) & in_block) * Kv4Tile::bytes(HD)); };
    uint64_t offsets = 0;
    int blocks_next = 0;
    if (n_it) offsets = offsets_of(0, table[tile_of_lane(0) >> a.tiles_shift]), blocks_next = table[tile_of_lane(64) >> a.tiles_shift];
    uint32_t codes[G], scales;
    auto load = [&](int it) {
        if (it && it % 64 == 0) {
            offsets = offsets_of(it, blocks_next);
            blocks_next = table[tile_of_lane(it + 64) >> a.tiles_shift];
        }
        const uint32_t lo32 = __builtin_amdgcn_readlane((uint32_t)offsets, it % 64), hi32 = __builtin_amdgcn_readlane((uint32_t)(offsets >> 32), it % 64);
        const PoolPtr at = base + ((uint64_t)hi32 << 32 | lo32);
        load_words<false, G>(at + (of_v ? Kv4Tile::v_codes(HD) : 0) + (uint32_t)lane * LB, codes);
        if (of_v) {
            scales = *(const EE_GLOBAL uint32_t*)(at + Kv4Tile::v_scales(HD) + (uint32_t)(t16 * EPC / 32 * 16 + quarter * 4));
        } else {
            scales = *(const EE_GLOBAL uint32_t*)(at + Kv4Tile::k_scales(HD) + (uint32_t)(t16 * G));
        }
    };
    auto convert = [&](int it, int buf) {
        if (of_v) {
            const int key0 = chunk_of(it) * KV4_CHUNK;
            if (key0 + KV4_CHUNK > pos_first + 1 || key0 < first_of(pos_last)) {
                // V behind the last position that any entry sees may hold anything: a scale of 1 makes it finite, and its
                // probabilities are zero.  NaN that not every entry sees is taken out here and put back by who sees it.
                const int key = key0 + 16 * tl + quarter * 4;
                uint32_t keep = 0, nan = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (key + i <= pos_last) keep |= 255u << (8 * i);
                    if ((scales >> (8 * i) & 255u) == SCALE_NAN) nan |= 255u << (8 * i);
                }
                nan &= keep;
                if (t16 * EPC % 32 == 0) s_scales[buf][tl][t16 * EPC / 32 * 4 + quarter] = nan;
                const bool any = __any(nan != 0);
                if (lane == 0) s_nan[buf][tl] = any;
                scales = (scales & keep & ~nan) | (0x7f7f7f7fu & (~keep | nan));
            }
            float unit[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) unit[i] = scale_of(scales, i);
            char* dst = (char*)&s_buffers[buf][KS * 64 + (tl * DB * 2 + (quarter & 1)) * 32 + t16] + (quarter >> 1) * 8;
#pragma unroll
            for (int b = 0; b < EPC / 2; ++b) {
                uint32_t x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int byte = i * (HD / 32) + b;
                    x[i] = pair_of(codes[byte >> 2], unit[i], byte & 3);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t sel = h ? 0x07060302u : 0x05040100u;
                    *(u32x2*)(dst + (b * 64 + h * 16) * 16) = u32x2{__builtin_amdgcn_perm(x[1], x[0], sel), __builtin_amdgcn_perm(x[3], x[2], sel)};
                }
            }
        } else {
            u32x4* dst = &s_buffers[buf][(quarter & 1) * 32 + tl * 16 + t16];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float unit = scale_of(scales, g);
                dst[(g * 2 + (quarter >> 1)) * 64] = u32x4{pair_of<0>(codes[g], unit), pair_of<1>(codes[g], unit), pair_of<2>(codes[g], unit), pair_of<3>(codes[g], unit)};
            }
        }
    };

    f32x16 o[DB] = {};
    float m = -INFINITY, l = 0.f, l_lse = 0.f;  // m: as above
    // The second group's matrix products come when the first one's vector work does: its scores are formed an interval ahead, so K
    // is converted two steps ahead there.
    const int ahead = group && !of_v ? 2 : 1;
    if (n_it) {
        load(0);
        convert(0, 0);
        if (n_it > 1) load(1);
        if (ahead == 2 && n_it > 1) {
            convert(1, 1);
            if (n_it > 2) load(2);
        }
    }
    f32x16 s;
    auto works = [&](int it) {
        const int key0 = chunk_of(it) * KV4_CHUNK;
        return !idle && it < n_it && key0 <= wave_last && key0 + KV4_CHUNK > first_of(wave_first);
    };
    auto scores = [&](int it) {  // rows = positions, columns = entries
        s = f32x16{};
#pragma unroll
        for (int k = 0; k < KS; ++k)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, s_buffers[it & 1][k * 64 + lane]), q[k], s, 0, 0, 0);
    };
    if (group) __builtin_amdgcn_s_setprio(1);  // (the younger waves of each SIMD, which it would serve last)
    __syncthreads();
    if (group && works(0)) scores(0);
    __syncthreads();
    for (int it = 0; it < n_most; ++it) {
        const int buf = it & 1, key0 = chunk_of(it) * KV4_CHUNK;
        if (works(it)) {
            if (!group) scores(it);
            // position of s[i]: key0 + 8 (i / 4) + 4 half + i % 4
            const bool wg_edge = key0 + KV4_CHUNK > pos_first + 1 || key0 < first_of(pos_last);
            if (key0 + KV4_CHUNK > wave_first + 1 || key0 < first_of(wave_last)) {
                int key = key0 + 4 * half;
                asm volatile("" : "+v"(key));
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int k = key + 8 * (i >> 2) + (i & 3);
                    if (k > hi || k < lo) s[i] = -INFINITY;
                }
            }
            float top = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
            float t0, t1;
            halves_of(top, t0, t1);
            top = fmaxf(fmaxf(t0, t1), m);
            if (__any(top > m + a.slack)) {
                const float corr = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - top) * a.scale_log2);
                l *= corr;
                if constexpr (LSE) l_lse *= corr;
#pragma unroll
                for (int b = 0; b < DB; ++b) o[b] *= corr;
                m = top;
            }
            const float ref = m == -INFINITY ? 0.f : m * a.scale_log2;
            u32x4 p[2];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                f32x2 x;
                x[0] = __builtin_amdgcn_exp2f(fmaf(s[i], a.scale_log2, -ref));
                x[1] = __builtin_amdgcn_exp2f(fmaf(s[i + 1], a.scale_log2, -ref));
                const uint32_t rounded = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
                l = add_pair(rounded, l);
                if constexpr (LSE) l_lse += x[0] + x[1];
                p[i >> 3][(i & 7) >> 1] = rounded;
            }
            // weighted sum: rows = elements, columns = entries
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int b = 0; b < DB; ++b)
                    o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, s_buffers[buf][(KS + t * DB + b) * 64 + lane]),
                                                                   __builtin_bit_cast(bf16x8, p[t]), o[b], 0, 0, 0);
            if (wg_edge && (s_nan[buf][0] | s_nan[buf][1])) {
                // as in the kernel above: "is NaN" times "is seen", counted per column of V and entry
                f32x16 count = {};
                int key = key0 + 4 * half;
                asm volatile("" : "+v"(key));
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const uint32_t* sc = &s_scales[buf][t][t16 * EPC / 32 * 4];
                    bf16x8 is_nan, seen;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int k = key + 16 * t + 8 * (e >> 2) + (e & 3);
                        is_nan[e] = (__bf16)((sc[half + 2 * (e >> 2)] >> (8 * (e & 3)) & 255u) ? 1.f : 0.f);
                        seen[e] = (__bf16)(k <= hi && k >= lo ? 1.f : 0.f);
                    }
                    count = __builtin_amdgcn_mfma_f32_32x32x16_bf16(is_nan, seen, count, 0, 0, 0);
                }
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (count[i] > 0.f) o[b][i] = __builtin_nanf("");
            }
        }
        if (it + ahead < n_it) convert(it + ahead, (it + ahead) & 1);
        if (it + ahead + 1 < n_it) load(it + ahead + 1);
        if (group && works(it + 1)) scores(it + 1);
        __syncthreads();
    }

    // the second group's sums join the first's
    float* s_sums = (float*)s_operands;
    if (group) {
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) s_sums[((wave * DB + b) * 16 + i) * 64 + lane] = o[b][i];
        s_ml[0][wave * 64 + lane] = m, s_ml[1][wave * 64 + lane] = l;
        if constexpr (LSE) s_ml[2][wave * 64 + lane] = l_lse;
    }
    __syncthreads();
    if (!group) {
        const float m2 = s_ml[0][wave * 64 + lane], top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
        const float w1 = __builtin_amdgcn_exp2f((m - ref) * a.scale_log2), w2 = __builtin_amdgcn_exp2f((m2 - ref) * a.scale_log2);
        l = l * w1 + s_ml[1][wave * 64 + lane] * w2;
        if constexpr (LSE) l_lse = l_lse * w1 + s_ml[2][wave * 64 + lane] * w2;
        m = top;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][i] = o[b][i] * w1 + s_sums[((wave * DB + b) * 16 + i) * 64 + lane] * w2;
    }
    float l0, l1;
    halves_of(l, l0, l1);
    const float sum = l0 + l1;
    float sum_lse = 0.f;
    if constexpr (LSE) {
        halves_of(l_lse, l0, l1);
        sum_lse = l0 + l1;
    }
    if (!group && f_wave + col < f_end) {
        const size_t r = (size_t)(w.row0 + row) * (a.group * a.kv_heads) + head, at = (size_t)w.slot * M + 32 * wave + col;
        const float inv = 1.f / sum;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const PartPlace<HD, 512, M> place(wave, i);
            const int c = place.column;  // of V: elements c * EPC ...
            if (n_parts == 1) {
                uint32_t x[EPC / 2];
#pragma unroll
                for (int b = 0; b < DB; ++b)
                    x[b] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{o[b][i] * inv, o[b][8 + i] * inv}, bf16x2));
                *(u32x4*)(out + r * HD + c * EPC) = u32x4{x[0], x[1], x[2], x[3]};
            } else {
#pragma unroll
                for (int b = 0; b < DB; ++b) hand_over2(a.part_o + (size_t)w.slot * (M * HD) + place.held(b), f32x2{o[b][i], o[b][8 + i]});
            }
        }
        if (half == 0) {
            if (n_parts > 1) {
                hand_over2(a.part_ml + 2 * at, f32x2{m * a.scale_log2, sum});
                if constexpr (LSE) hand_over1(a.part_l + at, sum_lse);
            } else if constexpr (LSE) {
                a.lse[r] = ((m == -INFINITY ? 0.f : m * a.scale_log2) + log2f(sum_lse)) * 0.6931471805599453f;
            }
        }
    }
    if (n_parts > 1) join_parts<HD, 512, M, LSE, __bf16>(a, w, n_parts, f0, f_end, &s_last);
}

template <int HD, int UNITS, int NW>
hipError_t attend_waves(const Kv4Attend& a, int dtype, int grid, hipStream_t s) {
    // (tiles of more than 16 entries: a request has several, which read the same K and V.  With 256 elements all tiles have 16,
    // so a prompt's tiles there read them past the caches as well: 1024 rows at 8192 positions, 16 heads on 4, 237 us, its
    // products 106)
    const bool past = UNITS == 1 && a.past_caches;
    // Two steps ahead where registers allow it at the same number of waves: 8 waves alone on a CU, and bf16 tiles of 32 entries (17
    // requests of 500 to 12 560 positions and 15 rows, 32 heads on 8: 61 us, one step ahead 64; 64 of 500 to 16 384 and 5 rows: 144
    // and 163).
    constexpr int DEPTH = NW == 8 && HD <= 128 ? 2 : 1, DEPTH_BF16 = UNITS == 2 && HD <= 128 ? 2 : DEPTH;
    const dim3 g(grid), t(NW * 64);
    if constexpr (UNITS <= 2)
        if (dtype == EE_F32) {
            EE_LAUNCH((past ? kv4_attend_kernel<HD, 3, 3, UNITS, NW, DEPTH, UNITS == 1, true, float>
                            : kv4_attend_kernel<HD, 3, 3, UNITS, NW, DEPTH, false, true, float>),
                      g, t, s, a);
            return hipGetLastError();
        }
    if constexpr (UNITS == 1)
        EE_LAUNCH((past ? kv4_attend_kernel<HD, 1, 2, 1, NW, DEPTH_BF16, true, true, __bf16> : kv4_attend_kernel<HD, 1, 2, 1, NW, DEPTH_BF16, false, true, __bf16>), g,
                  t, s, a);
    else
        EE_LAUNCH((a.lse ? kv4_attend_kernel<HD, 1, 1, UNITS, NW, DEPTH_BF16, false, true, __bf16>
                         : kv4_attend_kernel<HD, 1, 1, UNITS, NW, DEPTH_BF16, false, false, __bf16>),
                  g, t, s, a);
    return hipGetLastError();
}

template <int HD, int UNITS>
hipError_t attend_units(const Kv4Attend& a, int dtype, int waves, int grid, hipStream_t s) {
    if constexpr (UNITS == 1)
        if (waves == 8) return attend_waves<HD, 1, 8>(a, dtype, grid, s);
    return attend_waves<HD, UNITS, 4>(a, dtype, grid, s);
}

template <int HD>
hipError_t attend_hd(const Kv4Attend& a, int dtype, int units, int waves, int grid, hipStream_t s) {
    if (units == 1) return attend_units<HD, 1>(a, dtype, waves, grid, s);
    if constexpr (HD <= 128)
        if (units == 2) return attend_units<HD, 2>(a, dtype, waves, grid, s);
    if constexpr (HD == 128) {
        if (units == KV4_WIDE / 16 && dtype == EE_BF16) {
            EE_LAUNCH((a.lse ? kv4_attend_wide_kernel<true> : kv4_attend_wide_kernel<false>), dim3(grid), dim3(512), s, a);
            return hipGetLastError();
        }
    }
    if constexpr (HD <= 64)
        if (units == 4 && dtype == EE_BF16) return attend_units<HD, 4>(a, dtype, waves, grid, s);
    return hipErrorInvalidValue;
}

inline bool aligned16(const void* p, int64_t row, int64_t head, int es) {
    return ((uintptr_t)p & 15) == 0 && (row * es) % 16 == 0 && (head * es) % 16 == 0;
}

// rows of a launch: a grid has less than 2^32 threads (half as many here)
inline int rows_of_launch(int n_rows, int threads_per_row) { return std::min(n_rows, (int)((1ll << 31) / threads_per_row) & ~15); }

template <int HD>
hipError_t append_hd(const Kv4Cache& c, int n_rows, const void* k, int64_t k_row, int64_t k_head, const void* v, int64_t v_row, int64_t v_head,
                     const int64_t* slots, bool of_plan, hipStream_t s) {
    const int es = c.dtype == EE_BF16 ? 2 : 4;
    const int vec = (aligned16(k, k_row, k_head, es) ? 1 : 0) | (aligned16(v, v_row, v_head, es) ? 2 : 0);
    const int each = rows_of_launch(n_rows, c.kv_heads * 2 * 64 / 16);
    for (int row0 = 0; row0 < n_rows; row0 += each) {
        const int64_t waves = (int64_t)((std::min(each, n_rows - row0) + 15) / 16) * c.kv_heads * 2;
        const dim3 grid((unsigned)((waves + 3) / 4));
        if (c.dtype == EE_BF16)
            EE_LAUNCH((kv4_append_kernel<HD, __bf16>), grid, dim3(256), s, c, n_rows, (const __bf16*)k, k_row, k_head, (const __bf16*)v, v_row, v_head,
                      vec, slots, of_plan ? 0 : n_rows, row0);
        else
            EE_LAUNCH((kv4_append_kernel<HD, float>), grid, dim3(256), s, c, n_rows, (const float*)k, k_row, k_head, (const float*)v, v_row, v_head, vec,
                      slots, of_plan ? 0 : n_rows, row0);
    }
    return hipGetLastError();
}

template <int HD>
hipError_t read_hd(const Kv4Cache& c, int n_rows, const int64_t* slots, void* k, void* v, hipStream_t s) {
    const int per_row = c.kv_heads * 2 * (HD / 8), each = rows_of_launch(n_rows, per_row);
    for (int row0 = 0; row0 < n_rows; row0 += each) {
        const int64_t threads = (int64_t)((std::min(each, n_rows - row0) + 15) / 16 * 16) * per_row;
        const dim3 grid((unsigned)((threads + 255) / 256));
        if (c.dtype == EE_BF16)
            EE_LAUNCH((kv4_read_kernel<HD, __bf16>), grid, dim3(256), s, c, n_rows, slots, (__bf16*)k, (__bf16*)v, row0);
        else
            EE_LAUNCH((kv4_read_kernel<HD, float>), grid, dim3(256), s, c, n_rows, slots, (float*)k, (float*)v, row0);
    }
    return hipGetLastError();
}

}  // namespace

constexpr int64_t WIDE_ITEMS = 160;

bool kv4_has_wide_tiles(int dtype, int head_dim) { return dtype == EE_BF16 && head_dim == 128; }

int kv4_tile_units(int dtype, int head_dim, int most_flat, int n_seqs, int64_t all_flat, int kv_heads) {
    // Wide tiles, in which an element is converted once for 128 entries, where they give more than half of the CUs work (32
    // heads on 8, one request at 4000 positions: 520 rows, 130 tiles, 89 us, in tiles of 32 entries 72; 900 rows, 225 tiles, 81
    // and 87) and where not an eighth of them stays empty (24 requests of 500 to 4000 positions and 33 rows, 132 entries and
    // two tiles each: 98 and 75; 32 rows: 60 and 61).  Requests that do not all bring the most waste half a tile each on the
    // average.  A tile has a CU to itself, so a second round for a few of them costs as much as for all: 1024 rows at 8192
    // positions are 256 tiles and take 146 us, 1032 rows 262.  With 64 elements a wave holds 64 entries itself, and those tiles
    // are as good or better (20 heads on 4, a prompt of 4000 rows: 76 us, wide 91).
    if (kv4_has_wide_tiles(dtype, head_dim) && all_flat * kv_heads >= KV4_WIDE * WIDE_ITEMS) {
        const bool alike = (int64_t)n_seqs * most_flat <= all_flat;
        const int64_t empty = (int64_t)n_seqs * (alike ? (KV4_WIDE - most_flat % KV4_WIDE) % KV4_WIDE : KV4_WIDE / 2);
        if (empty * 8 <= all_flat) return KV4_WIDE / 16;
    }
    const int most = dtype == EE_BF16 ? std::min(4, 256 / head_dim) : std::min(2, 256 / head_dim);  // what a wave's registers hold
    int units = 1;
    while (units < most && 16 * units < most_flat) units *= 2;
    return units;
}

hipError_t launch_kv4_init(int32_t* table, int64_t n_table, int32_t* free_blocks, int n_blocks, uint32_t* arrived, int n_arrived,
                           uint32_t* counts, hipStream_t s) {
    EE_LAUNCH(kv4_init_kernel, dim3(1024), dim3(256), s, table, n_table, free_blocks, n_blocks, arrived, n_arrived, counts);
    return hipGetLastError();
}

hipError_t launch_kv4_plan(const Kv4Plan& p, int workgroups, int threads, hipStream_t s) {
    EE_LAUNCH(kv4_plan_kernel, dim3(workgroups), dim3(threads), s, p);
    return hipGetLastError();
}

hipError_t launch_kv4_append(const Kv4Cache& c, int n_rows, const void* k, int64_t k_row, int64_t k_head, const void* v, int64_t v_row,
                             int64_t v_head, const int64_t* slots, bool of_plan, hipStream_t s) {
    switch (c.head_dim) {
        case 32: return append_hd<32>(c, n_rows, k, k_row, k_head, v, v_row, v_head, slots, of_plan, s);
        case 64: return append_hd<64>(c, n_rows, k, k_row, k_head, v, v_row, v_head, slots, of_plan, s);
        case 128: return append_hd<128>(c, n_rows, k, k_row, k_head, v, v_row, v_head, slots, of_plan, s);
        case 256: return append_hd<256>(c, n_rows, k, k_row, k_head, v, v_row, v_head, slots, of_plan, s);
        default: return hipErrorInvalidValue;
    }
}

hipError_t launch_kv4_read(const Kv4Cache& c, int n_rows, const int64_t* slots, void* k, void* v, hipStream_t s) {
    switch (c.head_dim) {
        case 32: return read_hd<32>(c, n_rows, slots, k, v, s);
        case 64: return read_hd<64>(c, n_rows, slots, k, v, s);
        case 128: return read_hd<128>(c, n_rows, slots, k, v, s);
        case 256: return read_hd<256>(c, n_rows, slots, k, v, s);
        default: return hipErrorInvalidValue;
    }
}

hipError_t launch_kv4_attend(const Kv4Attend& a, int dtype, int head_dim, int units, int waves, int grid, hipStream_t s) {
    if (grid <= 0) return hipSuccess;
    switch (head_dim) {
        case 32: return attend_hd<32>(a, dtype, units, waves, grid, s);
        case 64: return attend_hd<64>(a, dtype, units, waves, grid, s);
        case 128: return attend_hd<128>(a, dtype, units, waves, grid, s);
        case 256: return attend_hd<256>(a, dtype, units, waves, grid, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace ee
