// The 4-bit paged cache (ee_kv4_* of ee.h): layout of a block, the plan's work list, and the launches.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "ee.h"

namespace ee {

// A layer of the pool is [n_blocks][n_kv_heads][block_tokens / 16] tiles of 16 positions of one head, 17 * head_dim bytes each,
// in the order in which a wave's lanes hold them for the matrix instructions, so that every load of a tile is one contiguous
// run of head_dim / 8 bytes per lane.  With G = head_dim / 32 groups and lane = 16 * quarter + column:
//   K codes   lane (quarter h, key t): G words, word g = elements 32g + 8h .. + 7 of key t, element e in bits 4e
//   V codes   lane (quarter h, column c): of keys 4h .. 4h+3, head_dim / 32 bytes each, elements c * head_dim / 16 ...
//   K scales  [16 keys][G] bytes, e + 127
//   V scales  [G][16 keys] bytes
// V lies by columns because the product P.V contracts over positions: a lane's word holds one position's elements of its own
// columns, and the conversion to bf16 is followed by one byte permute per two elements instead of a pass through LDS.
struct Kv4Tile {
    static constexpr int bytes(int hd) { return 17 * hd; }
    static constexpr int v_codes(int hd) { return 8 * hd; }
    static constexpr int k_scales(int hd) { return 16 * hd; }
    static constexpr int v_scales(int hd) { return 16 * hd + hd / 2; }
};

// multiplier for divisions by d > 1
inline uint32_t magic_of(uint32_t d) { return 0xffffffffu / d + 1; }

// One workgroup's share of the attention: part `part` of `n_parts` of the positions that one tile of rows of one kv head sees.
// A request's rows and the query heads that share a kv head form one list, row-major (entry f = row f / group, head f % group);
// a tile is the entries tile * M .. tile * M + M - 1.
struct Kv4Part {
    int32_t seq;     // request, -1: the rows see nothing
    int32_t row0;    // first row of the request
    int32_t n_flat;  // rows * group
    int32_t start;   // position of row0
    int32_t tile, head;
    int32_t part_of;  // part | n_parts << 16
    int32_t slot;     // where the part is left (the item's first part's slot + part) if there are several
};

struct Kv4Plan {
    const int32_t *held, *start, *end;
    int n_seqs, n_rows, max_rows_per_seq;
    int block_shift, n_blocks, table_stride, max_positions;  // 1 << block_shift positions per block
    ee_kv4_arrays a;
    Kv4Part* parts;
    int32_t* counts;    // [2]: parts, shape
    int32_t shape;      // plan_shape of its rows and tiles
    uint32_t* arrived;  // workgroups that have read the lengths
    int max_parts;  // room in `parts`
    int group, kv_heads, tile_rows, tile_shift;  // tile_rows = 1 << tile_shift
    uint32_t kv_magic;                           // magic_of(kv_heads)
    int target_parts;  // a launch is cut so that it has about this many parts
    int min_chunks;    // of a part that is one of several
    int whole_shares;  // an item is cut into as many parts as it has shares of the work, else into one more
};

// What calls of a plan's rows are launched for, and the plan leaves on the device: a captured call that is replayed after another
// plan would have too few rows of its arrays, or another size of tiles.
inline int32_t plan_shape(int n_rows, int tile_units) { return n_rows | tile_units << 24; }  // (n_rows <= 2^20, tile_units <= 8)

struct Kv4Cache {
    char* layer;  // this layer's pool
    int kv_heads, head_dim, block_shift, dtype;  // 1 << block_shift positions per block
    int64_t n_slots;
    const int32_t* counts;  // the plan's
};

struct Kv4Attend {
    const char* layer;
    const int32_t* table;
    int table_stride;
    const Kv4Part* parts;
    const int32_t* counts;  // the plan's
    int32_t shape, grid;  // of the launch
    const void* q;
    int64_t q_row, q_head;
    void* out;
    float* lse;
    float scale_log2;  // scale / ln 2
    float slack;       // scores that differ by this have probabilities that differ by 2^8 (finite however small the scale is)
    int window, group, kv_heads;
    uint32_t group_magic;  // magic_of(group)
    int min_chunks;  // of a part that is one of several
    int tiles_shift;  // log2(block_tokens / 16)
    int past_caches;  // K and V are read without keeping them in the caches
    int q_vec;        // rows of q can be read 16 bytes at a time
    float* part_o;    // [slot][tile rows][head_dim]
    float *part_ml, *joined_ml;  // [slot][tile rows][2]: reference and sum; of parts; of groups of parts, at the first one's slot
    float *part_l, *joined_l;    // [slot][tile rows]: sums for the log-sum-exp, where they are apart
    uint32_t *arrived, *arrived_groups;  // [slot] of the first part of a group, of an item: parts, groups that have been left
};

constexpr int KV4_WIDE = 128;  // entries of the tiles of prompts
constexpr int KV4_CHUNK = 32;  // positions: what a wave works on at a time, and the grain of the parts

// Entries of a tile in units of 16 (the columns of a matrix instruction), by the most that a request has for one kv head, and by
// what all requests may have for one.
int kv4_tile_units(int dtype, int head_dim, int most_flat, int n_seqs, int64_t all_flat, int kv_heads);
bool kv4_has_wide_tiles(int dtype, int head_dim);

hipError_t launch_kv4_init(int32_t* table, int64_t n_table, int32_t* free_blocks, int n_blocks, uint32_t* arrived, int n_arrived,
                           uint32_t* counts, hipStream_t s);
hipError_t launch_kv4_plan(const Kv4Plan& p, int workgroups, int threads, hipStream_t s);
hipError_t launch_kv4_append(const Kv4Cache& c, int n_rows, const void* k, int64_t k_row, int64_t k_head, const void* v, int64_t v_row,
                             int64_t v_head, const int64_t* slots, bool of_plan, hipStream_t s);
hipError_t launch_kv4_read(const Kv4Cache& c, int n_rows, const int64_t* slots, void* k, void* v, hipStream_t s);
hipError_t launch_kv4_attend(const Kv4Attend& a, int dtype, int head_dim, int units, int waves, int grid, hipStream_t s);

}  // namespace ee
