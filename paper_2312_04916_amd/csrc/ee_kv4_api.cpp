// Host side of the 4-bit paged cache (ee_kv4_* of ee.h): buffer layout, argument checks, and how a step's attention is cut.
#include <algorithm>
#include <cmath>
#include <new>

#include "ee_internal.h"
#include "ee_kv4.h"

using namespace ee;

namespace {

inline size_t align_up(size_t v, size_t a = 256) { return (v + a - 1) / a * a; }

int check_config(const ee_kv4_config& c) {
    if (c.n_layers < 1 || c.n_layers > 1024 || c.n_kv_heads < 1 || c.n_heads < 1 || c.n_heads > 1024 || c.n_heads % c.n_kv_heads)
        return EE_ERR_CONFIG;
    if (c.head_dim != 32 && c.head_dim != 64 && c.head_dim != 128 && c.head_dim != 256) return EE_ERR_CONFIG;
    if (c.dtype != EE_F32 && c.dtype != EE_BF16) return EE_ERR_CONFIG;
    if (c.block_tokens < 16 || c.block_tokens > 256 || (c.block_tokens & (c.block_tokens - 1))) return EE_ERR_CONFIG;
    if (c.n_blocks < 1 || c.n_blocks > (1 << 26)) return EE_ERR_CONFIG;
    if (c.max_seqs < 1 || c.max_seqs > EE_KV4_MAX_SEQS) return EE_ERR_CONFIG;
    if (c.max_positions < 1 || c.max_positions > (1 << 20)) return EE_ERR_CONFIG;
    if (c.max_rows < 1 || c.max_rows > (1 << 20)) return EE_ERR_CONFIG;
    return EE_OK;
}

// How a launch of the attention is cut: workgroups of `waves` waves, in about `parts` parts of at least `min_chunks` chunks; whole:
// an item is cut into as many parts as it has shares of the work (else into one more, so that none is longer than a share).
constexpr int MOST_PARTS = 768;
struct Cut {
    int waves, parts, min_chunks;
    bool whole;
};
int most_of_cut(int units) { return units * 16 == KV4_WIDE ? 256 : MOST_PARTS; }
Cut cut_of(const ee_kv4_config& c, int n_seqs, int n_rows, int units) {
    if (units * 16 == KV4_WIDE) return {8, most_of_cut(units), 32, true};
    if (units == 1) {
        // few items: one workgroup of eight waves per CU (one request of 131 071 positions, 8 kv heads: 32 us, with three of four
        // waves 43; 4 of 8000: 12.0, 15.7); many are balanced better by the smaller ones (64 of up to 16 384: 115, with eight
        // waves 151; 16 of up to 2048, 32 heads: 20, 24).  A request counts as one tile, though with 256 elements, where all tiles
        // are of 16 entries, one with many rows has more
        const int items = std::min(n_seqs, n_rows) * c.n_kv_heads;
        if (items < 128) return {8, 256, 8, true};
        return {4, MOST_PARTS, 8, false};
    }
    // Larger tiles leave as many times more to be joined, and a CU holds two workgroups.  So few items are cut into no more parts
    // than there are CUs (40 rows at 4000 positions, 32 heads on 8: 16 us, with 512 parts 22.5, with 768 27), some into two per
    // CU (17 requests of 500 to 12 560 and 15 rows: 61 us, with 256 parts 113, with 768 68), and many, which fill the chip uncut,
    // so that the longest do not end last (61 requests of up to 16 380 and 0 to 10 rows: 132, with 512 parts 169).
    const int64_t items = ((int64_t)n_rows * (c.n_heads / c.n_kv_heads) / (16 * units) + std::min(n_seqs, n_rows)) * c.n_kv_heads;
    if (items <= 128) return {4, 256, 8, true};
    if (items <= 512) return {4, 512, 8, true};
    return {4, MOST_PARTS, 8, false};
}

// A pool of more than half of the last-level cache (256 MB) is not found there again by the next step, which has read weights in
// between: keeping what is read only pushes other data out (589 MB of 64 requests: 114 us, kept 124; where the pool fits, keeping is
// the faster: 113 MB of 16 requests 30 us, past the caches 32).
constexpr size_t PAST_CACHES_BYTES = 128u << 20;

int table_stride(const ee_kv4_config& c) { return (c.max_positions + c.block_tokens - 1) / c.block_tokens; }
size_t layer_bytes(const ee_kv4_config& c) {
    return (size_t)c.n_blocks * c.n_kv_heads * (c.block_tokens / 16) * Kv4Tile::bytes(c.head_dim);
}

// Workgroups that a step's attention takes at most: one per item (tile of rows, kv head), the parts beyond that, and the tiles
// that are not full (one per request that has rows, one behind the last).
int64_t most_parts(const ee_kv4_config& c, int n_seqs, int n_rows, int tile_rows) {
    const int64_t tiles = (int64_t)n_rows * (c.n_heads / c.n_kv_heads) / tile_rows + std::min(n_seqs, n_rows) + 1;
    return tiles * c.n_kv_heads + MOST_PARTS + 64;  // (64: the share is formed in fp32)
}

struct StateLayout {
    size_t table, free_blocks, slots, positions, row_seq, row_start, served, held_next, counts, parts, arrived, part_ml, part_o, total;
    int64_t max_parts;
    int max_slots, part_rows;  // parts of items that are cut, and their rows: each of these has more than half its full length, so
                               // twice the target bounds them
};

StateLayout state_layout(const ee_kv4_config& c) {
    StateLayout w;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t o = off;
        off += align_up(bytes);
        return o;
    };
    w.table = take((size_t)c.max_seqs * table_stride(c) * 4);
    w.free_blocks = take((size_t)c.n_blocks * 4);
    w.slots = take((size_t)c.max_rows * 8);
    w.positions = take((size_t)c.max_rows * 4);
    w.row_seq = take((size_t)c.max_rows * 4);
    w.row_start = take(((size_t)c.max_seqs + 1) * 4);
    w.served = take((size_t)c.max_seqs * 4);
    w.held_next = take((size_t)c.max_seqs * 4);
    w.counts = take(16);  // free blocks, the plan's workgroups that have read the lengths, parts, the plan's shape
    w.max_parts = most_parts(c, c.max_seqs, c.max_rows, 16);
    w.parts = take((size_t)w.max_parts * sizeof(Kv4Part));
    w.max_slots = 2 * MOST_PARTS + 64;
    w.arrived = take((size_t)w.max_slots * 8);  // of groups of parts, of items
    // (of the largest tiles of one wave, or of wide ones)
    const int units = kv4_tile_units(c.dtype, c.head_dim, 64, 1, 0, c.n_kv_heads);
    w.part_rows = (2 * most_of_cut(units) + 64) * 16 * units;
    if (kv4_has_wide_tiles(c.dtype, c.head_dim)) w.part_rows = std::max(w.part_rows, (2 * most_of_cut(KV4_WIDE / 16) + 64) * KV4_WIDE);
    w.part_ml = take((size_t)w.part_rows * 24);  // of parts, of joined ones; then the log-sum-exp's of both
    w.part_o = take((size_t)w.part_rows * c.head_dim * 4);
    w.total = off;
    return w;
}

int hip_status(hipError_t e) { return e == hipSuccess ? EE_OK : ee::note_hip_error((int)e); }

}  // namespace

struct ee_kv4 {
    ee_kv4_config cfg;
    char *pool, *state;
    StateLayout sl;
    int n_seqs, n_rows, units, waves, min_chunks;  // of the latest plan (n_seqs = 0: none)
    ee_kv4_arrays arrays;
};

extern "C" {

int ee_kv4_bytes(const ee_kv4_config* cfg, size_t* pool_bytes, size_t* state_bytes) {
    if (!cfg) return EE_ERR_ARG;
    const int rc = check_config(*cfg);
    if (rc != EE_OK) return rc;
    if (pool_bytes) *pool_bytes = layer_bytes(*cfg) * cfg->n_layers;
    if (state_bytes) *state_bytes = state_layout(*cfg).total;
    return EE_OK;
}

int ee_kv4_create(const ee_kv4_config* cfg, void* dev_pool, size_t pool_bytes, void* dev_state, size_t state_bytes, void* stream,
                  ee_kv4** out) {
    if (!cfg || !dev_pool || !dev_state || !out) return EE_ERR_ARG;
    if (((uintptr_t)dev_pool | (uintptr_t)dev_state) & 255) return EE_ERR_ARG;
    size_t pb, sb;
    const int rc = ee_kv4_bytes(cfg, &pb, &sb);
    if (rc != EE_OK) return rc;
    if (pool_bytes < pb || state_bytes < sb) return EE_ERR_NOMEM;
    ee_kv4* c = new (std::nothrow) ee_kv4();
    if (!c) return EE_ERR_NOMEM;
    c->cfg = *cfg;
    c->pool = (char*)dev_pool;
    c->state = (char*)dev_state;
    c->sl = state_layout(*cfg);
    c->n_seqs = c->n_rows = 0;
    c->units = 1, c->waves = 4, c->min_chunks = 8;
    const StateLayout& w = c->sl;
    ee_kv4_arrays& a = c->arrays;
    a.table = (int32_t*)(c->state + w.table);
    a.free_blocks = (int32_t*)(c->state + w.free_blocks);
    a.slots = (int64_t*)(c->state + w.slots);
    a.positions = (int32_t*)(c->state + w.positions);
    a.row_seq = (int32_t*)(c->state + w.row_seq);
    a.row_start = (int32_t*)(c->state + w.row_start);
    a.served = (int32_t*)(c->state + w.served);
    a.held_next = (int32_t*)(c->state + w.held_next);
    a.n_free = (int32_t*)(c->state + w.counts);
    a.table_stride = table_stride(*cfg);
    const int st = hip_status(launch_kv4_init(a.table, (int64_t)cfg->max_seqs * a.table_stride, a.free_blocks, cfg->n_blocks,
                                              (uint32_t*)(c->state + w.arrived), 2 * w.max_slots, (uint32_t*)a.n_free, (hipStream_t)stream));
    if (st != EE_OK) {
        delete c;
        return st;
    }
    *out = c;
    return EE_OK;
}

int ee_kv4_free(ee_kv4* c) {
    if (!c) return EE_ERR_ARG;
    delete c;
    return EE_OK;
}

int ee_kv4_get_arrays(const ee_kv4* c, ee_kv4_arrays* out) {
    if (!c || !out) return EE_ERR_ARG;
    *out = c->arrays;
    return EE_OK;
}

int ee_kv4_plan(ee_kv4* c, int n_seqs, const int32_t* dev_held, const int32_t* dev_start, const int32_t* dev_end, int n_rows,
                int max_rows_per_seq, void* stream) {
    if (!c || !dev_held || !dev_start || !dev_end) return EE_ERR_ARG;
    if (((uintptr_t)dev_held | (uintptr_t)dev_start | (uintptr_t)dev_end) & 3) return EE_ERR_ARG;
    const ee_kv4_config& g = c->cfg;
    if (n_seqs < 1 || n_seqs > g.max_seqs || n_rows < 0 || n_rows > g.max_rows || max_rows_per_seq < 0) return EE_ERR_ARG;
    const int group = g.n_heads / g.n_kv_heads;
    const int most = std::min(max_rows_per_seq, n_rows);
    Kv4Plan p;
    p.held = dev_held, p.start = dev_start, p.end = dev_end;
    p.n_seqs = n_seqs, p.n_rows = n_rows, p.max_rows_per_seq = most;
    p.block_shift = __builtin_ctz((unsigned)g.block_tokens), p.n_blocks = g.n_blocks, p.table_stride = c->arrays.table_stride, p.max_positions = g.max_positions;
    p.a = c->arrays;
    p.parts = (Kv4Part*)(c->state + c->sl.parts);
    p.arrived = (uint32_t*)c->arrays.n_free + 1;
    p.counts = c->arrays.n_free + 2;
    p.group = group, p.kv_heads = g.n_kv_heads;
    const int units = kv4_tile_units(g.dtype, g.head_dim, (int)std::min<int64_t>((int64_t)most * group, 1 << 30), n_seqs, (int64_t)n_rows * group,
                                     g.n_kv_heads);
    p.shape = plan_shape(n_rows, units);
    p.tile_rows = 16 * units, p.tile_shift = __builtin_ctz((unsigned)p.tile_rows), p.kv_magic = magic_of((uint32_t)g.n_kv_heads);
    p.max_parts = (int)std::min(c->sl.max_parts, most_parts(g, n_seqs, n_rows, p.tile_rows));
    const Cut cut = cut_of(g, n_seqs, n_rows, units);
    p.target_parts = cut.parts, p.min_chunks = cut.min_chunks, p.whole_shares = cut.whole;
    // one thread per row and part, and for blocks that change hands, which only the GPU knows, an eighth of the pool; a small
    // step in one small workgroup
    const int threads = n_seqs < 256 && n_rows <= 1024 ? 256 : 1024;
    const int64_t tasks = (int64_t)n_rows + p.max_parts + g.n_blocks / 8;
    const int workgroups = n_rows + p.max_parts <= 2048 && g.n_blocks <= 4096 && threads == 256 ? 1 : (int)std::min<int64_t>(256, 1 + tasks / threads);
    const int rc = hip_status(launch_kv4_plan(p, workgroups, threads, (hipStream_t)stream));
    if (rc != EE_OK) return rc;
    c->n_seqs = n_seqs, c->n_rows = n_rows, c->units = units, c->waves = cut.waves, c->min_chunks = cut.min_chunks;
    return EE_OK;
}

static int check_rows(const ee_kv4* c, int layer, int n_rows) {
    if (!c) return EE_ERR_ARG;
    if (layer < 0 || layer >= c->cfg.n_layers) return EE_ERR_RANGE;
    if (n_rows < 0 || n_rows > (1 << 22)) return EE_ERR_ARG;
    return EE_OK;
}

static Kv4Cache geometry(const ee_kv4* c, int layer) {
    Kv4Cache k;
    k.layer = c->pool + layer_bytes(c->cfg) * layer;
    k.kv_heads = c->cfg.n_kv_heads, k.head_dim = c->cfg.head_dim, k.block_shift = __builtin_ctz((unsigned)c->cfg.block_tokens), k.dtype = c->cfg.dtype;
    k.n_slots = (int64_t)c->cfg.n_blocks * c->cfg.block_tokens;
    k.counts = c->arrays.n_free + 2;
    return k;
}

int ee_kv4_append(ee_kv4* c, int layer, int n_rows, const void* dev_k, int64_t k_row_stride, int64_t k_head_stride, const void* dev_v,
                  int64_t v_row_stride, int64_t v_head_stride, const int64_t* dev_slots, void* stream) {
    const int rc = check_rows(c, layer, n_rows);
    if (rc != EE_OK) return rc;
    if (!dev_slots && c->n_seqs == 0) return EE_ERR_STATE;
    if (!dev_slots && n_rows > c->n_rows) return EE_ERR_ARG;
    if (n_rows == 0) return EE_OK;
    const uintptr_t es = c->cfg.dtype == EE_BF16 ? 2 : 4;
    if (!dev_k || !dev_v || ((uintptr_t)dev_k | (uintptr_t)dev_v) & (es - 1) || (uintptr_t)dev_slots & 7) return EE_ERR_ARG;
    return hip_status(launch_kv4_append(geometry(c, layer), n_rows, dev_k, k_row_stride, k_head_stride, dev_v, v_row_stride, v_head_stride,
                                        dev_slots ? dev_slots : c->arrays.slots, !dev_slots, (hipStream_t)stream));
}

int ee_kv4_read(ee_kv4* c, int layer, int n_rows, const int64_t* dev_slots, void* dev_k, void* dev_v, void* stream) {
    const int rc = check_rows(c, layer, n_rows);
    if (rc != EE_OK) return rc;
    if (n_rows == 0) return EE_OK;
    if (!dev_slots || (!dev_k && !dev_v) || ((uintptr_t)dev_k | (uintptr_t)dev_v) & 15 || (uintptr_t)dev_slots & 7) return EE_ERR_ARG;
    return hip_status(launch_kv4_read(geometry(c, layer), n_rows, dev_slots, dev_k, dev_v, (hipStream_t)stream));
}

int ee_kv4_attend(ee_kv4* c, int layer, const void* dev_q, int64_t q_row_stride, int64_t q_head_stride, void* dev_out, float* dev_lse,
                  float scale, int window, void* stream) {
    const int rc = check_rows(c, layer, 0);
    if (rc != EE_OK) return rc;
    if (c->n_seqs == 0) return EE_ERR_STATE;
    const float scale_log2 = (scale > 0.f ? scale : 1.f / std::sqrt((float)c->cfg.head_dim)) * 1.4426950408889634f;
    if (!(scale >= 0.f) || std::isinf(scale_log2) || window < 0) return EE_ERR_ARG;
    if (c->n_rows == 0) return EE_OK;
    const ee_kv4_config& g = c->cfg;
    const uintptr_t es = g.dtype == EE_BF16 ? 2 : 4;
    if (!dev_q || !dev_out || (uintptr_t)dev_q & (es - 1) || (uintptr_t)dev_out & 15 || (uintptr_t)dev_lse & 3) return EE_ERR_ARG;
    // rows of q are read while others' results are already written
    const int64_t rows_span = (c->n_rows - 1) * q_row_stride, heads_span = (g.n_heads - 1) * q_head_stride, es_i = (int64_t)es;
    const uintptr_t q_lo = (uintptr_t)dev_q + (uintptr_t)(es_i * (std::min<int64_t>(rows_span, 0) + std::min<int64_t>(heads_span, 0)));
    const uintptr_t q_hi = (uintptr_t)dev_q + (uintptr_t)(es_i * (std::max<int64_t>(rows_span, 0) + std::max<int64_t>(heads_span, 0) + g.head_dim));
    const size_t results = (size_t)c->n_rows * g.n_heads;
    auto overlaps = [&](const void* p, size_t bytes) { return p && (uintptr_t)p < q_hi && q_lo < (uintptr_t)p + bytes; };
    if (overlaps(dev_out, results * g.head_dim * es) || overlaps(dev_lse, results * 4)) return EE_ERR_ARG;
    Kv4Attend a;
    a.layer = c->pool + layer_bytes(g) * layer;
    a.table = c->arrays.table, a.table_stride = c->arrays.table_stride;
    a.parts = (const Kv4Part*)(c->state + c->sl.parts);
    a.counts = c->arrays.n_free + 2;
    a.shape = plan_shape(c->n_rows, c->units);
    a.q = dev_q, a.q_row = q_row_stride, a.q_head = q_head_stride;
    a.out = dev_out, a.lse = dev_lse;
    a.scale_log2 = scale_log2;
    a.slack = std::min(8.f / scale_log2, 1e30f);
    a.window = window, a.group = g.n_heads / g.n_kv_heads, a.kv_heads = g.n_kv_heads, a.min_chunks = c->min_chunks;
    a.group_magic = magic_of((uint32_t)a.group);
    a.tiles_shift = __builtin_ctz((unsigned)g.block_tokens) - 4;
    a.past_caches = layer_bytes(g) * g.n_layers > PAST_CACHES_BYTES;
    a.q_vec = ((uintptr_t)dev_q & 15) == 0 && (q_row_stride * (int64_t)es) % 16 == 0 && (q_head_stride * (int64_t)es) % 16 == 0;
    a.part_o = (float*)(c->state + c->sl.part_o);
    a.part_ml = (float*)(c->state + c->sl.part_ml);
    a.joined_ml = a.part_ml + (size_t)c->sl.part_rows * 2;
    a.part_l = a.joined_ml + (size_t)c->sl.part_rows * 2;
    a.joined_l = a.part_l + c->sl.part_rows;
    a.arrived = (uint32_t*)(c->state + c->sl.arrived);
    a.arrived_groups = a.arrived + c->sl.max_slots;
    a.grid = (int)std::min(c->sl.max_parts, most_parts(g, c->n_seqs, c->n_rows, 16 * c->units));
    return hip_status(launch_kv4_attend(a, g.dtype, g.head_dim, c->units, c->waves, a.grid, (hipStream_t)stream));
}

}  // extern "C"
