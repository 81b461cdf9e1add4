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
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t SCALE_NAN = 255;              // of a group that stands for NaN
constexpr uint32_t SCALE_MIN = 16, SCALE_MAX = 252;  // 2^-111, 2^125: no held value is subnormal or infinite in bf16

// ------------------------------------------------------------------------------------------------
// create
// ------------------------------------------------------------------------------------------------
__global__ void kv4_init_kernel(int32_t* table, int64_t n_table, int32_t* free_blocks, int n_blocks, uint32_t* arrived, int n_arrived) {
    const int64_t i0 = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = i0; i < n_table; i += step) table[i] = 0;
    for (int64_t i = i0; i < n_blocks; i += step) free_blocks[i] = n_blocks - 1 - (int)i;  // block 0 is on top
    for (int64_t i = i0; i < n_arrived; i += step) arrived[i] = 0;
}

// ------------------------------------------------------------------------------------------------
// plan
// ------------------------------------------------------------------------------------------------
constexpr int PLAN_SEQS = EE_KV4_MAX_SEQS + 1;  // and the rows behind the last request's

// Sums over a workgroup: exclusive prefix of each thread's value, and the total.
template <int N>
__device__ void scan_sums(int64_t (&v)[N], int64_t (&total)[N], int64_t (*wave_sums)[N]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_waves = blockDim.x >> 6;
    int64_t own[N];
#pragma unroll
    for (int k = 0; k < N; ++k) own[k] = v[k];
    for (int d = 1; d < 64; d <<= 1) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int64_t o = __shfl_up(v[k], d);
            if (lane >= d) v[k] += o;
        }
    }
    __syncthreads();  // (wave_sums may still be read from the scan before)
    if (lane == 63) {
#pragma unroll
        for (int k = 0; k < N; ++k) wave_sums[wave][k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        int64_t before = 0, all = 0;
        for (int w = 0; w < n_waves; ++w) {
            const int64_t s = wave_sums[w][k];
            before += w < wave ? s : 0;
            all += s;
        }
        v[k] += before - own[k];
        total[k] = all;
    }
}

// Last index i < n with first[i] <= x (first ascending, first[0] <= x): of several equal ones the last, which is the one that
// is not empty.
__device__ __forceinline__ int last_not_above(const int32_t* first, int n, int32_t x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// Every workgroup forms the sums over all requests for itself (a few thousand lengths at most: cheaper than handing them on)
// and takes its share of the rows, blocks and parts.  What a workgroup reads, no other one writes: a block that one request
// gives back and another one takes is looked up in the table row of the first, behind what it keeps, which nothing changes.
// (dev_held == held_next is the one exception, and the launch then has one workgroup.)
__global__ __launch_bounds__(1024) void kv4_plan_kernel(Kv4Plan p) {
    __shared__ int32_t s_row[PLAN_SEQS];   // first row
    __shared__ int32_t s_take[PLAN_SEQS];  // blocks taken by the requests before; then first part
    __shared__ int32_t s_give[PLAN_SEQS];  // blocks given back by the requests before; then parts per item << 16 | served
    __shared__ int64_t s_sums[16][4];
    const int tid = threadIdx.x, nt = blockDim.x;
    const int n = p.n_seqs, per = (n + 1 + nt - 1) / nt;
    const int i0 = min(n, tid * per), i1 = min(n, i0 + per);
    const int bt = p.block_tokens;
    const bool first_wg = blockIdx.x == 0;

    struct Req {
        int held, start, end, had, need, rows;
        bool ok;
    };
    auto request = [&](int i) {
        Req r;
        r.held = p.held[i], r.start = p.start[i], r.end = p.end[i];
        const int most = p.max_positions;
        const bool range = r.start >= 0 && r.start <= r.end && r.end <= most;
        r.ok = range && r.held >= 0 && r.held <= most && r.end - r.start <= p.max_rows_per_seq;
        r.rows = range ? r.end - r.start : 0;
        r.had = (min(max(r.held, 0), most) + bt - 1) / bt;
        r.need = r.ok ? (r.end + bt - 1) / bt : r.had;
        return r;
    };

    // blocks held, given back, asked for; rows
    int64_t v[4] = {0, 0, 0, 0}, all[4];
    for (int i = i0; i < i1; ++i) {
        const Req r = request(i);
        v[0] += r.had, v[1] += max(r.had - r.need, 0), v[2] += max(r.need - r.had, 0), v[3] += r.rows;
    }
    scan_sums<4>(v, all, s_sums);
    const int left = (int)max((int64_t)0, p.n_blocks - all[0]);  // free before the call (< 0: the lengths contradict the pool)
    const int have = left + (int)all[1];
    const int rows_all = (int)min(all[3], (int64_t)p.n_rows);
    // a request whose rows do not fit is refused, and gives and takes nothing: only then do the sums have to be formed again
    // (rows_all is what the caller says it is, unless its lengths are wrong)
    const bool clipped = all[3] > p.n_rows;
    if (clipped) {
        int64_t row = v[3];
        int64_t w[2] = {0, 0}, all2[4];
        for (int i = i0; i < i1; ++i) {
            const Req r = request(i);
            if (row + r.rows <= p.n_rows) w[0] += max(r.had - r.need, 0), w[1] += max(r.need - r.had, 0);
            row += r.rows;
        }
        int64_t x[4] = {w[0], w[1], 0, 0};
        scan_sums<4>(x, all2, s_sums);
        v[1] = x[0], v[2] = x[1];
        all[1] = all2[0], all[2] = all2[1];
    }
    const int have_now = clipped ? left + (int)all[1] : have;

    // per request: first row, blocks before it, served; and the work of its rows in chunks of positions
    int64_t work[4] = {0, 0, 0, 0}, work_all[4];
    {
        int64_t give = v[1], take = v[2], row = v[3];
        for (int i = i0; i < i1; ++i) {
            Req r = request(i);
            const bool fits = row + r.rows <= p.n_rows;
            if (!fits) r.ok = false, r.need = r.had;
            const int asked = max(r.need - r.had, 0);
            const bool ok = r.ok && (asked == 0 || take + asked <= have_now);
            s_row[i] = (int)min(row, (int64_t)p.n_rows);
            s_take[i] = (int)min(take, (int64_t)have_now);
            s_give[i] = (int)give;
            give += max(r.had - r.need, 0), take += asked;
            const int64_t row_end = row + r.rows;
            const int64_t tiles = ((min(row_end, (int64_t)p.n_rows) - min(row, (int64_t)p.n_rows)) * p.group + p.tile_rows - 1) / p.tile_rows;
            if (ok) work[0] += tiles * p.kv_heads * ((r.end + KV4_CHUNK - 1) / KV4_CHUNK);
            work[1] += asked > 0 && ok ? asked : 0;
            row = row_end;
            if (first_wg) {
                p.a.served[i] = ok ? 1 : 0;
                p.a.row_start[i] = s_row[i];
            }
        }
        if (tid == 0) s_row[n] = rows_all;
    }
    scan_sums<4>(work, work_all, s_sums);  // (its barriers also make s_row, s_take, s_give whole)
    const int taken = (int)work_all[1];
    const int chunks_per_part = (int)max((int64_t)p.min_chunks, (work_all[0] + p.target_parts - 1) / p.target_parts);

    auto served_of = [&](int i, const Req& r) {
        if (!r.ok) return false;
        const int asked = max(r.need - r.had, 0);
        // (s_take is capped at the blocks there are: a request behind the cap that asks for any is refused)
        return asked == 0 || (int64_t)s_take[i] + asked <= have_now;
    };
    auto request_at = [&](int i) {  // as above, with the rows that do not fit
        Req r = request(i);
        if (s_row[i] + (int64_t)r.rows > p.n_rows) r.ok = false, r.need = r.had, r.rows = p.n_rows - s_row[i];
        return r;
    };
    // entry `at` of the stack as it stands once everything given back lies on it
    auto stack = [&](int at) {
        if (at < left) return p.a.free_blocks[at];
        const int back = (int)all[1] - 1 - (at - left);  // in the requests' order, first block first
        const int i = last_not_above(s_give, n, back);
        const Req r = request_at(i);
        return p.a.table[(size_t)i * p.table_stride + min(r.need + back - s_give[i], p.table_stride - 1)];
    };

    const int64_t t0 = (int64_t)blockIdx.x * nt + tid, t_step = (int64_t)gridDim.x * nt;
    // rows
    for (int64_t r = t0; r < p.n_rows; r += t_step) {
        int64_t slot = -1;
        int pos = -1, seq = -1;
        if (r < rows_all) {
            seq = last_not_above(s_row, n, (int)r);
            const Req q = request_at(seq);
            if (served_of(seq, q)) {
                pos = q.start + (int)r - s_row[seq];
                const int b = pos / bt;
                const int block = b < q.had ? p.a.table[(size_t)seq * p.table_stride + b] : stack(have_now - 1 - (s_take[seq] + b - q.had));
                slot = (int64_t)block * bt + pos % bt;
            }
        }
        p.a.slots[r] = slot;
        p.a.positions[r] = pos;
        p.a.row_seq[r] = seq;
    }
    // blocks that are taken (n > 0 here: something was asked for)
    for (int64_t t = t0; t < taken; t += t_step) {
        const int i = last_not_above(s_take, n, (int)t);
        const Req q = request_at(i);
        const int b = q.had + (int)t - s_take[i];
        if (b < p.table_stride) p.a.table[(size_t)i * p.table_stride + b] = stack(have_now - 1 - (int)t);
    }
    // blocks that are given back
    for (int64_t t = t0; t < all[1]; t += t_step)
        if (left + t < p.n_blocks) p.a.free_blocks[left + t] = stack(left + (int)t);
    __syncthreads();

    // parts: items (tile of rows, kv head) in the requests' order, each cut alike; the rows behind the last request's are one
    // more "request" that sees nothing
    int64_t cnt[4] = {0, 0, 0, 0}, cnt_all[4];
    const int j1 = tid * per + per > n ? min(n + 1, tid * per + per) : i1;
    auto items_of = [&](int i, int& np, bool& sees, Req& r) {
        int flat;
        if (i < n) {
            r = request_at(i);
            sees = served_of(i, r) && r.rows > 0;
            flat = r.rows * p.group;
        } else {
            sees = false, flat = (p.n_rows - rows_all) * p.group, r.start = 0, r.rows = p.n_rows - rows_all;
        }
        np = sees ? ((r.end + KV4_CHUNK - 1) / KV4_CHUNK + chunks_per_part - 1) / chunks_per_part : 1;
        return (flat + p.tile_rows - 1) / p.tile_rows * p.kv_heads;
    };
    for (int i = min(n + 1, tid * per); i < j1; ++i) {
        int np;
        bool sees;
        Req r;
        const int items = items_of(i, np, sees, r);
        cnt[0] += (int64_t)items * np;
        cnt[1] += np > 1 ? (int64_t)items * np : 0;
    }
    scan_sums<4>(cnt, cnt_all, s_sums);
    for (int i = min(n + 1, tid * per); i < j1; ++i) {  // s_take, s_give: first part, first slot from here on
        int np;
        bool sees;
        Req r;
        const int items = items_of(i, np, sees, r);
        const int64_t first = cnt[0], slot = cnt[1];
        cnt[0] += (int64_t)items * np;
        cnt[1] += np > 1 ? (int64_t)items * np : 0;
        // (items_of reads s_take of request i only: this thread's own)
        s_take[i] = (int)first;
        s_give[i] = sees ? (int)slot : -1;
    }
    if (first_wg && tid == 0) {
        *p.n_parts = (int)min(cnt_all[0], (int64_t)p.max_parts);
        *p.a.n_free = have_now - taken;
        p.a.row_start[n] = rows_all;
    }
    __syncthreads();
    for (int64_t t = t0; t < min(cnt_all[0], (int64_t)p.max_parts); t += t_step) {
        const int i = last_not_above(s_take, n + 1, (int)t);
        Kv4Part w;
        const int local = (int)t - s_take[i];
        int np = 1, rows;
        w.start = 0;
        if (i < n) {
            const Req r = request_at(i);
            rows = r.rows;
            w.start = r.start;
            if (s_give[i] >= 0) np = ((r.end + KV4_CHUNK - 1) / KV4_CHUNK + chunks_per_part - 1) / chunks_per_part;
        } else {
            rows = p.n_rows - rows_all;
        }
        const int item = local / np;
        w.seq = s_give[i] >= 0 ? i : -1;
        w.row0 = s_row[i];
        w.n_flat = rows * p.group;
        // the tiles that see most come first
        const int tiles = (w.n_flat + p.tile_rows - 1) / p.tile_rows;
        w.tile = tiles - 1 - item / p.kv_heads;
        w.head = item % p.kv_heads;
        w.part_of = (local % np) | np << 16;
        w.slot = s_give[i] + local;
        p.parts[t] = w;
    }
    if (first_wg) {
        // (behind every read of the lengths: dev_held may be this array)
        __syncthreads();
        for (int i = i0; i < i1; ++i) p.a.held_next[i] = p.a.served[i] ? p.end[i] : p.held[i];
    }
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

__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false));  // lane ^ 1
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false));  // lane ^ 2
}

// tile of a slot's position, and the position in it
template <int HD>
__device__ __forceinline__ char* tile_of(const Kv4Cache& c, int64_t slot, int head, int& key) {
    const int64_t block = slot / c.block_tokens;
    const int in = (int)(slot % c.block_tokens);
    key = in & 15;
    return c.layer + ((block * c.kv_heads + head) * (c.block_tokens >> 4) + (in >> 4)) * (int64_t)Kv4Tile::bytes(HD);
}

// One thread per 8 elements, four threads per group: the largest magnitude by two lane exchanges, the conversion by the
// hardware's (which rounds to nearest even and saturates).
template <int HD, typename ST>
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4Cache c, int n_rows, const ST* __restrict__ k, int64_t k_row, int64_t k_head,
                                                         const ST* __restrict__ v, int64_t v_row, int64_t v_head, int vec,
                                                         const int64_t* __restrict__ slots) {
    constexpr int TPV = HD / 8, LB = HD / 8;  // threads per vector, bytes per lane of a tile
    const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int e8 = (int)(idx % TPV);
    const int64_t vecs = idx / TPV;
    const int which = (int)(vecs & 1), head = (int)((vecs >> 1) % c.kv_heads);
    const int64_t row = (vecs >> 1) / c.kv_heads;
    if (row >= n_rows) return;  // (whole groups of four lanes: their exchanges stay among themselves)
    const int64_t slot = slots[row];
    if (slot < 0 || slot >= c.n_slots) return;
    float x[8];
    const ST* src = which ? v + row * v_row + head * v_head : k + row * k_row + head * k_head;
    load8(src + e8 * 8, (vec >> which) & 1, x);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
    top = quad_max(top);
    // the least e with top <= 7 * 2^e = 1.75 * 2^(e+2); biased by 127
    uint32_t sc = min(max((top >> 23) + ((top & 0x7fffffu) > 0x600000u ? 1u : 0u), SCALE_MIN + 2) - 2, SCALE_MAX);
    const float unit = __uint_as_float(sc << 23);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], unit, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], unit, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], unit, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], unit, 3);
    if (top >= 0x7f800000u) sc = SCALE_NAN;
    int key;
    char* tile = tile_of<HD>(c, slot, head, key);
    const int g = e8 >> 2;
    if (which == 0) {
        *(uint32_t*)(tile + ((e8 & 3) * 16 + key) * LB + g * 4) = w;
        if ((e8 & 3) == 0) tile[Kv4Tile::k_scales(HD) + key * (HD / 32) + g] = (char)sc;
    } else {
        constexpr int EPC = HD / 16;  // elements per column
        char* t = tile + Kv4Tile::v_codes(HD) + (key & 3) * (LB / 4);
        const int col = (key >> 2) * 16 + e8 * 8 / EPC;
        if constexpr (EPC == 16) *(uint32_t*)(t + col * LB + (e8 & 1) * 4) = w;
        if constexpr (EPC == 8) *(uint32_t*)(t + col * LB) = w;
        if constexpr (EPC == 4) {
            *(uint16_t*)(t + col * LB) = (uint16_t)w;
            *(uint16_t*)(t + (col + 1) * LB) = (uint16_t)(w >> 16);
        }
        if constexpr (EPC == 2) {
#pragma unroll
            for (int b = 0; b < 4; ++b) t[(col + b) * LB] = (char)(w >> (8 * b));
        }
        if ((e8 & 3) == 0) tile[Kv4Tile::v_scales(HD) + g * 16 + key] = (char)sc;
    }
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
                                                       ST* __restrict__ v) {
    constexpr int TPV = HD / 8, LB = HD / 8;
    const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int e8 = (int)(idx % TPV);
    const int64_t vecs = idx / TPV;
    const int which = (int)(vecs & 1), head = (int)((vecs >> 1) % c.kv_heads);
    const int64_t row = (vecs >> 1) / c.kv_heads;
    if (row >= n_rows) return;
    ST* dst = which ? v : k;
    if (!dst) return;
    dst += (row * c.kv_heads + head) * HD + e8 * 8;
    const int64_t slot = slots[row];
    uint32_t w = 0, sc = SCALE_MIN;
    if (slot >= 0 && slot < c.n_slots) {
        int key;
        const char* tile = tile_of<HD>(c, slot, head, key);
        const int g = e8 >> 2;
        if (which == 0) {
            w = *(const uint32_t*)(tile + ((e8 & 3) * 16 + key) * LB + g * 4);
            sc = (uint8_t)tile[Kv4Tile::k_scales(HD) + key * (HD / 32) + g];
        } else {
            constexpr int EPC = HD / 16;
            const char* t = tile + Kv4Tile::v_codes(HD) + (key & 3) * (LB / 4);
            const int col = (key >> 2) * 16 + e8 * 8 / EPC;
            if constexpr (EPC == 16) w = *(const uint32_t*)(t + col * LB + (e8 & 1) * 4);
            if constexpr (EPC == 8) w = *(const uint32_t*)(t + col * LB);
            if constexpr (EPC == 4) w = *(const uint16_t*)(t + col * LB) | (uint32_t) * (const uint16_t*)(t + (col + 1) * LB) << 16;
            if constexpr (EPC == 2) {
#pragma unroll
                for (int b = 0; b < 4; ++b) w |= (uint32_t)(uint8_t)t[(col + b) * LB] << (8 * b);
            }
            sc = (uint8_t)tile[Kv4Tile::v_scales(HD) + g * 16 + key];
        }
    }
    bf16x2 x[4];
    values8(w, sc, x);
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

template <int N>
__device__ __forceinline__ void load_words(const char* p, uint32_t (&w)[N]) {
    if constexpr (N == 1) {
        w[0] = *(const uint32_t*)p;
    } else if constexpr (N == 2) {
        const u32x2 x = *(const u32x2*)p;
        w[0] = x[0], w[1] = x[1];
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const u32x4 x = *(const u32x4*)(p + 4 * i);
            w[i] = x[0], w[i + 1] = x[1], w[i + 2] = x[2], w[i + 3] = x[3];
        }
    }
}

template <int HD>
__device__ __forceinline__ void load_keys(const char* tile, int lane, KeyRegs<HD>& r) {
    constexpr int LB = HD / 8, G = HD / 32;
    load_words<G>(tile + lane * LB, r.w);
    const char* sc = tile + Kv4Tile::k_scales(HD) + (lane & 15) * G;
    if constexpr (G == 1) r.sc[0] = *(const uint8_t*)sc;
    if constexpr (G == 2) r.sc[0] = *(const uint16_t*)sc;
    if constexpr (G >= 4) load_words<G / 4>(sc, r.sc);
}
template <int HD>
__device__ __forceinline__ void load_values(const char* tile, int lane, ValueRegs<HD>& r) {
    constexpr int LB = HD / 8, G = HD / 32;
    load_words<G>(tile + Kv4Tile::v_codes(HD) + lane * LB, r.w);
    r.sc = *(const uint32_t*)(tile + Kv4Tile::v_scales(HD) + (lane & 15) * HD / 512 * 16 + (lane >> 4) * 4);
}

__device__ __forceinline__ float scale_of(const uint32_t* words, int i) {  // byte i as 2^(byte - 127)
    return __uint_as_float((words[i >> 2] >> (8 * (i & 3)) & 255u) << 23);
}

__device__ __forceinline__ uint32_t bytes_255(uint32_t w) {  // 0x80 in every byte of w that is 255 (and maybe above such a one)
    const uint32_t x = ~w;
    return (x - 0x01010101u) & ~x & 0x80808080u;
}

// What one workgroup leaves for another one of the same launch, maybe on another XCD.
__device__ __forceinline__ void hand_over(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float handed(const float* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// NT: bf16 terms of an element of Q (1: Q is bf16; 3: fp32, exactly), PT: of a probability.  UNITS: 16 entries each of a tile.
template <int HD, int NT, int PT, int UNITS, int NW, typename ST>
__global__ __launch_bounds__(NW * 64, (UNITS == 1 && HD <= 128) ? (NT == 1 ? 4 : 3) : 1) void kv4_attend_kernel(Kv4Attend a) {
    constexpr int G = HD / 32, EPC = HD / 16, M = 16 * UNITS;
    constexpr int CT = 2, STEPS = KV4_CHUNK / (16 * CT);  // tiles of 16 positions at a time: one contraction of P.V
    constexpr int LDO = HD + 4;
    __shared__ float s_o[NW * 16 * LDO];
    __shared__ float s_m[NW * 16], s_l[NW * 16];
    __shared__ uint32_t s_last;

    if ((int)blockIdx.x >= *a.n_parts) return;
    const Kv4Part w = a.parts[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const int f0 = w.tile * M, f_end = min(w.n_flat, f0 + M);  // entries
    const int n_heads = a.group * a.kv_heads;
    ST* out = (ST*)a.out;
    if (w.seq < 0) {
        for (int i = threadIdx.x; i < (f_end - f0) * HD; i += NW * 64) {
            const int f = f0 + i / HD;
            const size_t o = (size_t)(w.row0 + f / a.group) * n_heads + w.head * a.group + f % a.group;
            out[o * HD + i % HD] = (ST)0.f;
            if (i % HD == 0 && a.lse) a.lse[o] = -INFINITY;
        }
        return;
    }

    // entry f0 + 16 u + col of this lane: row, position, first and last position it sees
    bf16x8 q[UNITS][NT][G];
    int lo[UNITS], hi[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        const int f = min(f0 + 16 * u + col, f_end - 1);  // (columns behind the last entry repeat it; nobody reads them)
        const int row = f / a.group, head = w.head * a.group + f % a.group;
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
    const int pos_first = w.start + f0 / a.group, pos_last = w.start + (f_end - 1) / a.group;
    const int lo_min = a.window ? max(0, pos_first - a.window + 1) : 0;
    const int lo_max = a.window ? max(0, pos_last - a.window + 1) : 0;
    const int c_first = lo_min / KV4_CHUNK, n_chunks = pos_last / KV4_CHUNK + 1 - c_first;
    const int n_parts = w.part_of >> 16, part = w.part_of & 0xffff;
    const int c_lo = c_first + (int)((int64_t)n_chunks * part / n_parts), c_hi = c_first + (int)((int64_t)n_chunks * (part + 1) / n_parts);

    const int32_t* table = a.table + (size_t)w.seq * a.table_stride;
    const int last_tile = pos_last >> 4;
    const size_t block_bytes = ((size_t)Kv4Tile::bytes(HD) << a.tiles_shift) * a.kv_heads;
    const char* base = a.layer + ((size_t)Kv4Tile::bytes(HD) << a.tiles_shift) * w.head;
    const int in_block = (1 << a.tiles_shift) - 1;

    // step `it` of this wave: tiles (c_lo + wave + it / STEPS * NW) * 4 + it % STEPS * CT ...; tiles behind the last one that is
    // seen repeat it (their positions are hidden)
    const int my_chunks = max(0, (c_hi - c_lo - wave + NW - 1) / NW);
    const int n_it = my_chunks * STEPS;
    auto tile_at = [&](int it, int t) { return (c_lo + wave + it / STEPS * NW) * (KV4_CHUNK / 16) + it % STEPS * CT + t; };
    // block numbers of the next 64 / CT steps, one per lane
    constexpr int AHEAD = 64 / CT;
    auto blocks_from = [&](int it) {
        const int t = min(tile_at(it + lane / CT, lane % CT), last_tile);
        return table[t >> a.tiles_shift];
    };
    int blocks = n_it ? blocks_from(0) : 0;
    auto tile_addr = [&](int it, int t) {
        const int tile = min(tile_at(it, t), last_tile);
        const int block = __builtin_amdgcn_readlane(blocks, it % AHEAD * CT + t);
        return base + (size_t)block * block_bytes + (size_t)(tile & in_block) * Kv4Tile::bytes(HD);
    };

    f32x4 o[UNITS][EPC];
    float m[UNITS], l[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        m[u] = -INFINITY, l[u] = 0.f;
#pragma unroll
        for (int j = 0; j < EPC; ++j) o[u][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // K of the next step is asked for as soon as K of this one has been used, V likewise: one set of registers, and with four
    // waves per SIMD always about 45 KB on their way to a CU
    KeyRegs<HD> kr[CT];
    ValueRegs<HD> vr[CT];
    const char* at[CT];
    if (n_it) {
#pragma unroll
        for (int t = 0; t < CT; ++t) at[t] = tile_addr(0, t);
#pragma unroll
        for (int t = 0; t < CT; ++t) load_keys<HD>(at[t], lane, kr[t]);
#pragma unroll
        for (int t = 0; t < CT; ++t) load_values<HD>(at[t], lane, vr[t]);
    }
    for (int it = 0; it < n_it; ++it) {
        const int key0 = tile_at(it, 0) * 16;
        // scores: rows = positions, columns = entries
        f32x4 s[UNITS][CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) {
#pragma unroll
            for (int u = 0; u < UNITS; ++u) s[u][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float unit = scale_of(kr[t].sc, g);
                const bf16x8 kf = frag(pair_of<0>(kr[t].w[g], unit), pair_of<1>(kr[t].w[g], unit), pair_of<2>(kr[t].w[g], unit),
                                       pair_of<3>(kr[t].w[g], unit));
#pragma unroll
                for (int u = 0; u < UNITS; ++u)
#pragma unroll
                    for (int n = NT - 1; n >= 0; --n) s[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[u][n][g], s[u][t], 0, 0, 0);
            }
        }
        const bool more = it + 1 < n_it;
        if (more) {
            if ((it + 1) % AHEAD == 0) blocks = blocks_from(it + 1);
#pragma unroll
            for (int t = 0; t < CT; ++t) at[t] = tile_addr(it + 1, t);
#pragma unroll
            for (int t = 0; t < CT; ++t) load_keys<HD>(at[t], lane, kr[t]);
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
            if (__any(top > m[u])) {
                const float corr = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m[u] - top) * a.scale_log2);
                l[u] *= corr;
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
                    // (with one term the sum is that of the rounded probabilities, so that the weights add up to one)
                    if (PT > 1) l[u] += p[0] + p[1];
#pragma unroll
                    for (int n = 0; n < PT; ++n) {
                        const uint32_t h = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
                        pf[u][n][t * 2 + (i >> 1)] = h;
                        const float h0 = __uint_as_float(h << 16), h1 = __uint_as_float(h & 0xffff0000u);
                        if (PT == 1) l[u] += h0 + h1;
                        if (n + 1 < PT) p[0] -= h0, p[1] -= h1;
                    }
                }
        }
        // weighted sum: rows = elements (column c of V's layout), columns = entries
        float u0[4], u1[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u0[i] = scale_of(&vr[0].sc, i), u1[i] = scale_of(&vr[1].sc, i);
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
            for (int t = 0; t < CT; ++t) load_values<HD>(at[t], lane, vr[t]);
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
    }

    // join the waves' shares, 16 entries at a time
    constexpr int EPT = 16 * HD / (NW * 64);  // elements per thread
    const int e0 = threadIdx.x * EPT, my_row = e0 / HD, my_d = e0 % HD;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        if (f0 + 16 * u >= f_end) break;
        const float lsum = rows4_sum(l[u]);
        if (u) __syncthreads();
        if (f0 + 16 * u + col < f_end) {
            float* dst = s_o + (wave * 16 + col) * LDO;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < EPC; ++j) dst[(quarter * 4 + i) * EPC + j] = o[u][j][i];
            if (quarter == 0) s_m[wave * 16 + col] = m[u] * a.scale_log2, s_l[wave * 16 + col] = lsum;
        }
        __syncthreads();
        const int f = f0 + 16 * u + my_row;
        if (f < f_end) {
            float top = -INFINITY, sum = 0.f, acc[EPT];
#pragma unroll
            for (int v = 0; v < NW; ++v) top = fmaxf(top, s_m[v * 16 + my_row]);
            const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int e = 0; e < EPT; ++e) acc[e] = 0.f;
#pragma unroll
            for (int v = 0; v < NW; ++v) {
                const float wt = __builtin_amdgcn_exp2f(s_m[v * 16 + my_row] - ref);
                sum += wt * s_l[v * 16 + my_row];
                // (a wave that saw nothing has weight zero and zeros)
#pragma unroll
                for (int e = 0; e < EPT; ++e) acc[e] += wt * s_o[(v * 16 + my_row) * LDO + my_d + e];
            }
            if (n_parts == 1) {
                const size_t r = (size_t)(w.row0 + f / a.group) * n_heads + w.head * a.group + f % a.group;
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
                for (int e = 0; e < EPT; ++e) out[r * HD + my_d + e] = (ST)(acc[e] * inv);
                if (a.lse && my_d == 0) a.lse[r] = (ref + log2f(sum)) * 0.6931471805599453f;
            } else {
                const size_t r = (size_t)w.slot * M + 16 * u + my_row;
#pragma unroll
                for (int e = 0; e < EPT; ++e) hand_over(a.part_o + r * HD + my_d + e, acc[e]);
                if (my_d == 0) hand_over(a.part_ml + 2 * r, top), hand_over(a.part_ml + 2 * r + 1, sum);
            }
        }
    }
    if (n_parts == 1) return;

    // the workgroup that leaves the last part of the item joins them, in their order.  The parts go past the caches of this
    // XCD (agent-scope stores and loads): a release fence instead would write the whole of its L2 back, which cost a launch of
    // 1024 parts 300 us
    const int slot0 = w.slot - part;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // each thread's stores have arrived before the workgroup is counted
    __syncthreads();
    if (threadIdx.x == 0) s_last = __hip_atomic_fetch_add(a.arrived + slot0, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if ((int)s_last != n_parts - 1) return;
    if (threadIdx.x == 0) __hip_atomic_store(a.arrived + slot0, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int i = threadIdx.x; i < (f_end - f0) * HD; i += NW * 64) {
        const int r = i / HD, d = i % HD, f = f0 + r;
        float top = -INFINITY, sum = 0.f, acc = 0.f;
        for (int v = 0; v < n_parts; ++v) top = fmaxf(top, handed(a.part_ml + 2 * ((size_t)(slot0 + v) * M + r)));
        const float ref = top == -INFINITY ? 0.f : top;
        for (int v = 0; v < n_parts; ++v) {
            const size_t at = (size_t)(slot0 + v) * M + r;
            const float wt = __builtin_amdgcn_exp2f(handed(a.part_ml + 2 * at) - ref);
            sum += wt * handed(a.part_ml + 2 * at + 1);
            acc += wt * handed(a.part_o + at * HD + d);
        }
        const size_t at = (size_t)(w.row0 + f / a.group) * n_heads + w.head * a.group + f % a.group;
        out[at * HD + d] = (ST)(sum == 0.f ? 0.f : acc / sum);
        if (a.lse && d == 0) a.lse[at] = (ref + log2f(sum)) * 0.6931471805599453f;
    }
}

template <int HD, int UNITS>
hipError_t attend_units(const Kv4Attend& a, int dtype, int grid, hipStream_t s) {
    constexpr int NW = 4;
    if (dtype == EE_BF16)
        EE_LAUNCH((kv4_attend_kernel<HD, 1, UNITS == 1 ? 2 : 1, UNITS, NW, __bf16>), dim3(grid), dim3(NW * 64), s, a);
    else if constexpr (UNITS <= 2)
        EE_LAUNCH((kv4_attend_kernel<HD, 3, 3, UNITS, NW, float>), dim3(grid), dim3(NW * 64), s, a);
    else
        return hipErrorInvalidValue;
    return hipGetLastError();
}

template <int HD>
hipError_t attend_hd(const Kv4Attend& a, int dtype, int units, int grid, hipStream_t s) {
    if (units == 1) return attend_units<HD, 1>(a, dtype, grid, s);
    if constexpr (HD <= 128)
        if (units == 2) return attend_units<HD, 2>(a, dtype, grid, s);
    if constexpr (HD <= 64)
        if (units == 4) return attend_units<HD, 4>(a, dtype, grid, s);
    return hipErrorInvalidValue;
}

inline bool aligned16(const void* p, int64_t row, int64_t head, int es) {
    return ((uintptr_t)p & 15) == 0 && (row * es) % 16 == 0 && (head * es) % 16 == 0;
}

template <int HD>
hipError_t append_hd(const Kv4Cache& c, int n_rows, const void* k, int64_t k_row, int64_t k_head, const void* v, int64_t v_row, int64_t v_head,
                     const int64_t* slots, hipStream_t s) {
    const int es = c.dtype == EE_BF16 ? 2 : 4;
    const int vec = (aligned16(k, k_row, k_head, es) ? 1 : 0) | (aligned16(v, v_row, v_head, es) ? 2 : 0);
    const int64_t threads = (int64_t)n_rows * c.kv_heads * 2 * (HD / 8);
    const dim3 grid((unsigned)((threads + 255) / 256));
    if (c.dtype == EE_BF16)
        EE_LAUNCH((kv4_append_kernel<HD, __bf16>), grid, dim3(256), s, c, n_rows, (const __bf16*)k, k_row, k_head, (const __bf16*)v, v_row, v_head,
                  vec, slots);
    else
        EE_LAUNCH((kv4_append_kernel<HD, float>), grid, dim3(256), s, c, n_rows, (const float*)k, k_row, k_head, (const float*)v, v_row, v_head, vec,
                  slots);
    return hipGetLastError();
}

template <int HD>
hipError_t read_hd(const Kv4Cache& c, int n_rows, const int64_t* slots, void* k, void* v, hipStream_t s) {
    const int64_t threads = (int64_t)n_rows * c.kv_heads * 2 * (HD / 8);
    const dim3 grid((unsigned)((threads + 255) / 256));
    if (c.dtype == EE_BF16)
        EE_LAUNCH((kv4_read_kernel<HD, __bf16>), grid, dim3(256), s, c, n_rows, slots, (__bf16*)k, (__bf16*)v);
    else
        EE_LAUNCH((kv4_read_kernel<HD, float>), grid, dim3(256), s, c, n_rows, slots, (float*)k, (float*)v);
    return hipGetLastError();
}

}  // namespace

int kv4_tile_units(int dtype, int head_dim, int most_flat) {
    const int most = dtype == EE_BF16 ? std::min(4, 256 / head_dim) : std::min(2, 256 / head_dim);  // what a wave's registers hold
    int units = 1;
    while (units < most && 16 * units < most_flat) units *= 2;
    return units;
}

hipError_t launch_kv4_init(int32_t* table, int64_t n_table, int32_t* free_blocks, int n_blocks, uint32_t* arrived, int n_arrived,
                           hipStream_t s) {
    EE_LAUNCH(kv4_init_kernel, dim3(1024), dim3(256), s, table, n_table, free_blocks, n_blocks, arrived, n_arrived);
    return hipGetLastError();
}

hipError_t launch_kv4_plan(const Kv4Plan& p, int workgroups, hipStream_t s) {
    EE_LAUNCH(kv4_plan_kernel, dim3(workgroups), dim3(1024), s, p);
    return hipGetLastError();
}

hipError_t launch_kv4_append(const Kv4Cache& c, int n_rows, const void* k, int64_t k_row, int64_t k_head, const void* v, int64_t v_row,
                             int64_t v_head, const int64_t* slots, hipStream_t s) {
    switch (c.head_dim) {
        case 32: return append_hd<32>(c, n_rows, k, k_row, k_head, v, v_row, v_head, slots, s);
        case 64: return append_hd<64>(c, n_rows, k, k_row, k_head, v, v_row, v_head, slots, s);
        case 128: return append_hd<128>(c, n_rows, k, k_row, k_head, v, v_row, v_head, slots, s);
        case 256: return append_hd<256>(c, n_rows, k, k_row, k_head, v, v_row, v_head, slots, s);
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

hipError_t launch_kv4_attend(const Kv4Attend& a, int dtype, int head_dim, int units, int grid, hipStream_t s) {
    if (grid <= 0) return hipSuccess;
    switch (head_dim) {
        case 32: return attend_hd<32>(a, dtype, units, grid, s);
        case 64: return attend_hd<64>(a, dtype, units, grid, s);
        case 128: return attend_hd<128>(a, dtype, units, grid, s);
        case 256: return attend_hd<256>(a, dtype, units, grid, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace ee
