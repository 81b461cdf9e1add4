// Kernels of products with weights held in 8 bits (ee_f8_* of ee.h; layouts in ee_f8.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "ee_exp.h"
#include "ee_f8.h"
#include "ee_lanes.h"
#include "ee_launch.h"

namespace ee {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// ------------------------------------------------------------------------------------------------
// the format
// ------------------------------------------------------------------------------------------------

// Exponent (e + 127) of a group whose largest magnitude has these bits: the least e with top <= 448 * 2^e, 448 = 1.75 * 2^8.  255: the
// group holds an infinity or a NaN.
__device__ __forceinline__ uint32_t exponent_of(uint32_t top) {
    const int e = (int)(top >> 23) - 8 + ((top & 0x7fffff) > 0x600000 ? 1 : 0);
    return top >= 0x7f800000u ? 255u : (uint32_t)min(max(e, 127 - 110), 127 + 120);
}
// 2^-e, to be multiplied by; exact where the product is at least 2^-126, and a product below that is far below the least step
__device__ __forceinline__ float unit_inverse(uint32_t e) { return __uint_as_float((254 - e) << 23); }

// Four elements, in units of 2^e, as four codes.  No value is above 448, so nothing saturates.
__device__ __forceinline__ int codes4(float a, float b, float c, float d) {
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
constexpr int CODES_NAN = 0x7f7f7f7f;

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// 32 neighbouring elements of a row as floats, zeros behind the n that there are; row[0] is there in any case.  Sixteen bytes at a time
// wherever the row begins, and behind its end the first or last element again, for no branch to wait at (element by element
// where rows are not aligned to 16 bytes, 16 rows by 1001 x 2003 took 17.6 us for 8.2, 8 rows by 1000 x 4001 17.8 for 7.8).
template <typename T>
__device__ __forceinline__ void load32(const T* row, int n, float (&v)[32]) {
    constexpr int PER = 16 / sizeof(T);
    typedef i32x4 loose_i32x4 __attribute__((aligned(2)));
    if (n >= 32) {
#pragma unroll
        for (int i = 0; i < 32 / PER; ++i) {
            const i32x4 a = *(const loose_i32x4*)(row + i * PER);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 2) {
                    v[i * 8 + j * 2] = __uint_as_float((uint32_t)a[j] << 16);
                    v[i * 8 + j * 2 + 1] = __uint_as_float((uint32_t)a[j] & 0xffff0000u);
                } else {
                    v[i * 4 + j] = __int_as_float(a[j]);
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = (float)row[max(min(i, n - 1), 0)];
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = i < n ? v[i] : 0.f;
    }
}

__device__ __forceinline__ uint32_t top_of(const float (&v)[32]) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) top = max(top, magnitude(v[i]));
    return top;
}
// largest over the four lanes that hold a row's group
__device__ __forceinline__ uint32_t top_of_quarters(uint32_t t) {
    const lanes_u32x2 a = __builtin_amdgcn_permlane16_swap(t, t, false, false);
    t = max(a[0], a[1]);
    const lanes_u32x2 b = __builtin_amdgcn_permlane32_swap(t, t, false, false);
    return max(b[0], b[1]);
}
__device__ __forceinline__ void codes_of(const float (&v)[32], uint32_t e, i32x8& c) {
    const float u = unit_inverse(min(e, 247u));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int q = codes4(v[4 * i] * u, v[4 * i + 1] * u, v[4 * i + 2] * u, v[4 * i + 3] * u);
        c[i] = e == 255 ? CODES_NAN : q;
    }
}
// the exponent that is stored for a group: of one that stands for NaN any will do
__device__ __forceinline__ uint32_t stored(uint32_t e) { return e == 255 ? 127 : e; }

__device__ __forceinline__ void store_fragment(char* f, int lane, const i32x8& c) {
    *(i32x4*)(f + lane * 16) = __builtin_shufflevector(c, c, 0, 1, 2, 3);
    *(i32x4*)(f + 1024 + lane * 16) = __builtin_shufflevector(c, c, 4, 5, 6, 7);
}
__device__ __forceinline__ i32x8 load_fragment(const char* f, int lane) {
    const i32x4 a = *(const i32x4*)(f + lane * 16), b = *(const i32x4*)(f + 1024 + lane * 16);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// A workgroup packs one block of 128 rows x 128 elements, a wave the 16 rows of a fragment.  Bound by memory: 50 304 x 4096 in bf16 are
// packed in 115 us (618 MB, 5.4 TB/s).
template <typename T>
__global__ __launch_bounds__(512) void f8_pack_kernel(F8Shape s, const T* w, int64_t w_row, const T* up, int64_t up_row, char* weight) {
    __shared__ uint32_t s_top[8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, step = blockIdx.x;
    const int row = (blockIdx.y * 8 + wave) * 16 + (lane & 15), k0 = step * 128 + (lane >> 4) * 32;
    const T* src = blockIdx.z ? up : w;
    float v[32];
    load32(src + (int64_t)min(row, s.n - 1) * (blockIdx.z ? up_row : w_row) + min(k0, s.k - 1), row < s.n ? s.k - k0 : 0, v);
    uint32_t top = top_of(v);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if (lane == 0) s_top[wave] = top;
    __syncthreads();
    for (int i = 0; i < 8; ++i) top = max(top, s_top[i]);
    const uint32_t e = exponent_of(top);
    const int tile = (blockIdx.y * 8 + wave) * (s.pair ? 2 : 1) + blockIdx.z;
    if (tile >= s.tiles()) return;
    i32x8 c;
    codes_of(v, e, c);
    const size_t f = (size_t)tile * s.steps() + step;
    store_fragment(weight + f * F8_FRAGMENT, lane, c);
    // (the row's rounding up is written too: by the last tile)
    if (lane == 0) {
        for (int i = tile; i < (tile == s.tiles() - 1 ? s.exponent_row() : tile + 1); ++i)
            weight[s.exponents() + (size_t)step * s.exponent_row() + i] = (char)stored(e);
    }
}

// Back into values.  Bound by its stores, 32 of one element a lane: 50 304 x 4096 into bf16 1010 us, 0.6 TB/s (a call for tests and checks).
template <typename T>
__global__ __launch_bounds__(64) void f8_unpack_kernel(F8Shape s, int up, const char* weight, T* w) {
    const int lane = threadIdx.x, step = blockIdx.y, row = blockIdx.x * 16 + (lane & 15), k0 = step * 128 + (lane >> 4) * 32;
    const int tile = blockIdx.x * (s.pair ? 2 : 1) + up;
    const i32x8 c = load_fragment(weight + ((size_t)tile * s.steps() + step) * F8_FRAGMENT, lane);
    const float unit = __uint_as_float((uint32_t)(uint8_t)weight[s.exponents() + (size_t)step * s.exponent_row() + tile] << 23);
    if (row >= s.n) return;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const int word = c[i / 4] >> (i % 4 * 8);
        if (k0 + i < s.k) w[(int64_t)row * s.k + k0 + i] = (T)(__builtin_amdgcn_cvt_f32_fp8(word, 0) * unit);
    }
}

// ------------------------------------------------------------------------------------------------
// rows into 8 bits: a wave makes the fragment of 16 rows x 128 elements, a group's largest element by two lane swaps.  Bound by memory
// where there is much (4096 x 4096 in bf16: 11.4 us, 4.4 TB/s), by launch and one load where there is little (61 x 11 008: 3.6).
// ------------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void f8_rows_kernel(F8Rows r, const T* x, int64_t x_row, int k, char* out) {
    const int lane = threadIdx.x & 63, step = blockIdx.y * 4 + (threadIdx.x >> 6), tile = blockIdx.x;
    if (step >= r.steps) return;
    const int row = tile * 16 + (lane & 15), k0 = step * 128 + (lane >> 4) * 32;
    float v[32];
    load32(x + (int64_t)min(row, r.m - 1) * x_row + min(k0, k - 1), row < r.m ? k - k0 : 0, v);
    const uint32_t e = exponent_of(top_of_quarters(top_of(v)));
    i32x8 c;
    codes_of(v, e, c);
    const size_t f = (size_t)tile * r.steps + step;
    store_fragment(out + f * F8_FRAGMENT, lane, c);
    if (lane < 16) out[r.exponents() + f * 16 + lane] = (char)stored(e);
}

// ------------------------------------------------------------------------------------------------
// products
// ------------------------------------------------------------------------------------------------

// The held values of a fragment in bf16, which all of them fit: operands of four instructions of 32 elements.
__device__ __forceinline__ void values_of(const i32x8& c, float unit, bf16x8 (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * i], unit, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * i], unit, true);
        const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * i + 1], unit, false);
        const bf16x2 e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * i + 1], unit, true);
        v[i] = bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
    }
}

// T: of the result.  __expf costs |g| 2^-23 of it, below a bf16's half step of 2^-9 by far for all g that leave anything (down to -88), but many of fp32's.
template <typename T>
__device__ __forceinline__ float silu(float g) {
    return g / (1.f + (sizeof(T) == 2 ? __expf(-g) : exp_of(-g)));
}

// Four neighbouring results of one row: rows that are added, rounding to the nearest.  Moved at once wherever the row begins (one by one where rows
// were not aligned, 1321 rows by 2603 x 1267 took 19.2 us for 14.0, with fp32 results 31.4 for 22.6).
template <typename T>
__device__ __forceinline__ void finish(const F8Product& p, int row, int col, f32x4 v) {
    if (row >= p.m || col >= p.n) return;
    T* y = (T*)p.y + row * p.y_row + col;
    const T* add = p.add ? (const T*)p.add + row * p.add_row + col : nullptr;
    typedef T T4 __attribute__((ext_vector_type(4)));
    typedef T4 loose_T4 __attribute__((aligned(2)));
    if (col + 3 < p.n) {
        if (add) {
            const T4 a = *(const loose_T4*)add;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += (float)a[i];
        }
        *(loose_T4*)y = T4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < p.n) y[i] = (T)(add ? v[i] + (float)add[i] : v[i]);
    }
}

// Eight of them.
template <typename T>
__device__ __forceinline__ void finish8(const F8Product& p, int row, int col, f32x4 a, f32x4 b) {
    if (row >= p.m || col >= p.n) return;
    if (col + 7 >= p.n) {
        finish<T>(p, row, col, a);
        finish<T>(p, row, col + 4, b);
        return;
    }
    typedef T T8 __attribute__((ext_vector_type(8)));
    typedef T8 loose_T8 __attribute__((aligned(2)));
    if (p.add) {
        const T8 v = *(const loose_T8*)((const T*)p.add + row * p.add_row + col);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] += (float)v[i], b[i] += (float)v[i + 4];
    }
    *(loose_T8*)((T*)p.y + row * p.y_row + col) = T8{(T)a[0], (T)a[1], (T)a[2], (T)a[3], (T)b[0], (T)b[1], (T)b[2], (T)b[3]};
}

struct HeldRows {};  // they are in the workspace

// What a workgroup needs in LDS that quantises m rows itself: codes as [step][half][quarter][row] of 16 bytes, exponents as [step][row].
__host__ __device__ constexpr size_t own_rows_bytes(int m, int steps) { return (size_t)m * steps * 129; }

template <typename X, int THREADS>
__device__ __forceinline__ void quantise_rows(const F8Product& p, int steps, char* codes) {
    uint8_t* exponents = (uint8_t*)codes + (size_t)p.m * steps * 128;
    const int quarter = threadIdx.x & 3;
    for (int i = threadIdx.x / 4; i < p.m * steps; i += THREADS / 4) {
        const int row = i / steps, step = i - row * steps, k0 = step * 128 + quarter * 32;
        float v[32];
        load32((const X*)p.x + row * p.x_row + min(k0, p.k - 1), p.k - k0, v);
        uint32_t top = top_of(v);
        top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xb1, 0xf, 0xf, false));  // of the four lanes: 1 0 3 2
        top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4e, 0xf, 0xf, false));  // 2 3 0 1
        const uint32_t e = exponent_of(top);
        i32x8 c;
        codes_of(v, e, c);
        char* at = codes + ((size_t)(step * 8 + quarter) * p.m + row) * 16;
        *(i32x4*)at = __builtin_shufflevector(c, c, 0, 1, 2, 3);
        *(i32x4*)(at + (size_t)p.m * 64) = __builtin_shufflevector(c, c, 4, 5, 6, 7);
        if (quarter == 0) exponents[step * p.m + row] = (uint8_t)stored(e);
    }
}

// Few rows: the weight comes straight from memory into the registers of the wave that multiplies it.  A wave computes 16 * MT rows of x by NT
// tiles of the weight in every W-th step of 128 elements, D steps ahead of which its loads are; the waves' sums are added up in
// LDS in their order.  T: of the result; bf16: the 8-bit instructions, which add eight products at a time in multiples of 2^-13 of the largest
// (1.5e-5 of a result on Gaussian rows, next to the 1.7e-3 of its own rounding: one in some 50 rounds to its other side, the error against 64 bits stays 0.00165); float:
// the held values go through the bf16 instructions, which keep every bit of a product.  X: HeldRows, or the type in which sixteen rows at most come, which every workgroup then
// quantises for itself, into LDS, while its first loads of the weight are on their way.
// Bound by the weight's bytes: 1 row by 50 304 x 4096 with fp32 results 38.6 us (5.3 TB/s), 1 row by 6144 x 2048 5.2 us, launch included, 16 rows
// by a pair of 11 008 x 4096 16.2 (5.6 TB/s), 61 rows by 4096 x 11 008 13.4 (3.4 TB/s: each step's x comes from L2 next to the weight).
template <typename T, typename X, int MT, int NT, int W, int D>
__global__ __launch_bounds__(W * 64) void f8_stream_kernel(F8Product p, F8Shape s, F8Rows r, int m_groups, int n_groups) {
    constexpr bool RAW = !__is_same(X, HeldRows);
    static_assert(!RAW || MT == 1, "rows that are quantised here");
    extern __shared__ __attribute__((aligned(16))) char dynamic[];  // own rows, then the waves' sums
    f32x4(*s_part)[MT * NT][64] = (f32x4(*)[MT * NT][64])dynamic;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // the groups of rows that take the same tiles of the weight follow one another on one XCD
    const int xcd = blockIdx.x & 7, turn = blockIdx.x >> 3, n_group = turn / m_groups * 8 + xcd, m_group = turn % m_groups;
    if (n_group >= n_groups) return;
    const int tile0 = n_group * NT, mt0 = m_group * MT, tiles = s.tiles(), steps = s.steps(), m_tiles = (p.m + 15) / 16;
    const int exponent_row = s.exponent_row(), mine = (steps - wave + W - 1) / W;
    f32x4 acc[MT][NT] = {};
    struct Step {
        i32x8 w[NT], x[MT];
        int we[NT], xe[MT];
    };
    const char *w_at[NT], *x_at[MT];
#pragma unroll
    for (int j = 0; j < NT; ++j) w_at[j] = p.weight + (size_t)min(tile0 + j, tiles - 1) * steps * F8_FRAGMENT;
#pragma unroll
    for (int i = 0; i < MT; ++i) x_at[i] = p.workspace + (size_t)min(mt0 + i, m_tiles - 1) * steps * F8_FRAGMENT;
    const char* x_exponents = p.workspace + r.exponents();
    auto load = [&](Step& b, int step) {
        if constexpr (!RAW) {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                b.x[i] = load_fragment(x_at[i] + (size_t)step * F8_FRAGMENT, lane);
                b.xe[i] = (uint8_t)x_exponents[((size_t)min(mt0 + i, m_tiles - 1) * steps + step) * 16 + (lane & 15)];
            }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            b.w[j] = load_fragment(w_at[j] + (size_t)step * F8_FRAGMENT, lane);
            b.we[j] = (uint8_t)p.weight[s.exponents() + (size_t)step * exponent_row + min(tile0 + j, tiles - 1)];
        }
    };
    const int own_row = min(lane & 15, p.m - 1);
    auto multiply = [&](Step& b, int i) {
        if constexpr (RAW) {
            const int step = wave + i * W;
            const char* at = dynamic + ((size_t)(step * 8 + (lane >> 4)) * p.m + own_row) * 16;
            const i32x4 lo = *(const i32x4*)at, hi = *(const i32x4*)(at + (size_t)p.m * 64);
            b.x[0] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            b.xe[0] = ((const uint8_t*)dynamic)[(size_t)p.m * steps * 128 + step * p.m + own_row];
        }
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.w[j], b.x[i], acc[i][j], 0, 0, 0, b.we[j], 0, b.xe[i]);
        } else {
            bf16x8 wv[NT][4], xv[4];
#pragma unroll
            for (int j = 0; j < NT; ++j) values_of(b.w[j], __uint_as_float((uint32_t)b.we[j] << 23), wv[j]);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                values_of(b.x[i], __uint_as_float((uint32_t)b.xe[i] << 23), xv);
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int h = 0; h < 4; ++h) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[j][h], xv[h], acc[i][j], 0, 0, 0);
            }
        }
    };
    Step ring[D];
#pragma unroll
    for (int d = 0; d < D; ++d) load(ring[d], min(wave + d * W, steps - 1));  // (what a wave has no step for is never multiplied)
    if constexpr (RAW) {
        quantise_rows<X, W * 64>(p, steps, dynamic);
        __syncthreads();
    }
    int i = 0;
    for (; i + 2 * D <= mine; i += D) {
#pragma unroll
        for (int d = 0; d < D; ++d) multiply(ring[d], i + d), load(ring[d], wave + (i + D + d) * W);
    }
    if (i + D <= mine) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            multiply(ring[d], i + d);
            if (i + D + d < mine) load(ring[d], wave + (i + D + d) * W);
        }
        i += D;
    }
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (i + d < mine) multiply(ring[d], i + d);
    if constexpr (RAW) __syncthreads();  // (the rows are read no more)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) s_part[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    auto sum = [&](int t) {
        f32x4 v = s_part[0][t][lane];
#pragma unroll
        for (int i = 1; i < W; ++i) v += s_part[i][t][lane];
        return v;
    };
    const int row = lane & 15, col = (lane >> 4) * 4;
    if (p.pair) {
        if constexpr (NT > 1) {
            for (int t = wave; t < MT * NT / 2; t += W) {
                const int i = t / (NT / 2), j = t % (NT / 2) * 2;
                const f32x4 g = sum(i * NT + j), u = sum(i * NT + j + 1);
                finish<T>(p, (mt0 + i) * 16 + row, (tile0 + j) / 2 * 16 + col, f32x4{silu<T>(g[0]) * u[0], silu<T>(g[1]) * u[1], silu<T>(g[2]) * u[2], silu<T>(g[3]) * u[3]});
            }
        }
    } else {
        for (int t = wave; t < MT * NT; t += W) finish<T>(p, (mt0 + t / NT) * 16 + row, (tile0 + t % NT) * 16 + col, sum(t));
    }
}

typedef const char __attribute__((address_space(1))) global_char;
typedef const void __attribute__((address_space(1))) global_void;
#define F8_LDS(p) ((__attribute__((address_space(3))) void*)(p))
// (as in the prompt phase: the compiler would let every read wait for all copies into LDS that are on their way)
#define F8_READ(dst, at, off) asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(dst) : "v"(at), "n"(off))
#define F8_READ_BYTE(dst, at, off) asm volatile("ds_read_u8 %0, %1 offset:%2" : "=v"(dst) : "v"(at), "n"(off))

template <int N>
__device__ __forceinline__ void wait_copies() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Many rows: a workgroup of 2 x 2 waves computes 64 * MI rows of x by 4 * NI tiles of the weight, a wave 32 * MI by 2 * NI tiles in
// instructions of 32 x 32 x 64.  Both operands come through LDS, copied past the registers in their own order, 64 elements of
// the contraction at a time, four such stages in turn (three where two workgroups share a CU); the next stage's operands are read while
// the products of this one run.  Bound by the matrix cores.
constexpr int XCDS = 8, XCD_CUS = 32, CUS = XCDS * XCD_CUS;
constexpr int tile_stages(int mi, int ni) { return mi * ni > 8 || mi * ni == 4 ? 4 : 3; }  // (two workgroups share a CU up to 8)
constexpr int tile_stage_bytes(int mi, int ni) { return 4 * (mi + ni) * 1024 + 1024; }
constexpr int tile_lds(int mi, int ni) {
    const int stages = tile_stages(mi, ni) * tile_stage_bytes(mi, ni), results = 4 * 32 * (32 * ni + 4) * 4;
    return stages > results ? stages : results;
}
template <typename T, int MI, int NI>
__device__ __forceinline__ void f8_tile(const F8Product& p, const F8Shape& s, const F8Rows& r, int tile0, int mt0, char* lds) {
    constexpr int WT = 4 * NI, XT = 4 * MI, FRAGS = WT + XT, STAGES = tile_stages(MI, NI);
    constexpr int EXPONENTS = FRAGS * 1024, STAGE = tile_stage_bytes(MI, NI);  // 256 bytes of x's, of the weight's, two unused copies of them
    constexpr int COPIES = FRAGS / 4 + 1;                             // of a wave
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wn = wave & 1, wm = wave >> 1;
    const int steps = s.steps(), m_tiles = (p.m + 15) / 16, halves = 2 * steps;
    // what this wave copies: fragments, 512 bytes of either half of each, and a kind of exponents
    global_char* from[FRAGS / 4];
#pragma unroll
    for (int i = 0; i < FRAGS / 4; ++i) {
        const int f = wave * (FRAGS / 4) + i;
        from[i] = (global_char*)(f < WT ? p.weight + (size_t)min(tile0 + f, s.tiles() - 1) * steps * F8_FRAGMENT
                                        : p.workspace + (size_t)min(mt0 + f - WT, m_tiles - 1) * steps * F8_FRAGMENT);
    }
    const bool of_x = (wave & 1) == 0;
    global_char* from_e = (global_char*)(of_x ? p.workspace + r.exponents() + (size_t)mt0 * steps * 16 : p.weight + s.exponents());
    const uint32_t e_step = of_x ? 16 : s.exponent_row(), at_lane = (lane >> 5) * 1024 + (lane & 31) * 16;
    const uint32_t e_lane = of_x ? (uint32_t)min(lane >> 2, m_tiles - 1 - mt0) * steps * 16 + (lane & 3) * 4 : (uint32_t)min(tile0 + lane * 4, s.exponent_row() - 4);
    auto copy_one = [&](int buffer, size_t on, uint32_t on_e, int i) {
        if (i < FRAGS / 4)
            __builtin_amdgcn_global_load_lds((global_void*)(from[min(i, FRAGS / 4 - 1)] + on + at_lane), F8_LDS(lds + buffer * STAGE + (wave * (FRAGS / 4) + i) * 1024), 16, 0, 0);
        else
            __builtin_amdgcn_global_load_lds((global_void*)(from_e + on_e + e_lane), F8_LDS(lds + buffer * STAGE + EXPONENTS + wave * 256), 4, 0, 0);
    };
    auto offset_of = [&](int half) { return (size_t)(half >> 1) * F8_FRAGMENT + (half & 1) * 512; };
    struct Operands {
        i32x4 w[NI][2], x[MI][2];
        int we[NI], xe[MI];
    };
    const unsigned lds0 = (unsigned)(size_t)F8_LDS(lds), row32 = lane & 31;
    const unsigned at = (row32 >> 4) * 1024 + (lane >> 5) * 256 + (row32 & 15) * 16;
    const unsigned at_w = lds0 + wn * (2 * NI) * 1024 + at, at_x = lds0 + (WT + wm * (2 * MI)) * 1024 + at;
    const unsigned at_we = lds0 + EXPONENTS + 256 + wn * (2 * NI) + (row32 >> 4), at_xe = lds0 + EXPONENTS + wm * (32 * MI) + row32;
    f32x16 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.f;
    auto read_w = [&](Operands& o, unsigned stage, int j) {
        switch (j) {
            case 0: F8_READ(o.w[0][0], at_w + stage, 0); F8_READ(o.w[0][1], at_w + stage, 512); F8_READ_BYTE(o.we[0], at_we + stage, 0); break;
            case 1: F8_READ(o.w[1][0], at_w + stage, 2048); F8_READ(o.w[1][1], at_w + stage, 2560); F8_READ_BYTE(o.we[1], at_we + stage, 2); break;
            case 2: if constexpr (NI > 2) { F8_READ(o.w[2][0], at_w + stage, 4096); F8_READ(o.w[2][1], at_w + stage, 4608); F8_READ_BYTE(o.we[2], at_we + stage, 4); } break;
            case 3: if constexpr (NI > 3) { F8_READ(o.w[3][0], at_w + stage, 6144); F8_READ(o.w[3][1], at_w + stage, 6656); F8_READ_BYTE(o.we[3], at_we + stage, 6); } break;
        }
    };
    auto read_x = [&](Operands& o, unsigned stage, int i) {
        switch (i) {
            case 0: F8_READ(o.x[0][0], at_x + stage, 0); F8_READ(o.x[0][1], at_x + stage, 512); F8_READ_BYTE(o.xe[0], at_xe + stage, 0); break;
            case 1: F8_READ(o.x[1][0], at_x + stage, 2048); F8_READ(o.x[1][1], at_x + stage, 2560); F8_READ_BYTE(o.xe[1], at_xe + stage, 32); break;
            case 2: if constexpr (MI > 2) { F8_READ(o.x[2][0], at_x + stage, 4096); F8_READ(o.x[2][1], at_x + stage, 4608); F8_READ_BYTE(o.xe[2], at_xe + stage, 64); } break;
            case 3: if constexpr (MI > 3) { F8_READ(o.x[3][0], at_x + stage, 6144); F8_READ(o.x[3][1], at_x + stage, 6656); F8_READ_BYTE(o.xe[3], at_xe + stage, 96); } break;
        }
    };
    auto landed = [&](Operands& o) {  // (products that use them do not move above this)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int j = 0; j < NI; ++j) asm volatile("" : "+v"(o.w[j][0]), "+v"(o.w[j][1]), "+v"(o.we[j]));
#pragma unroll
        for (int i = 0; i < MI; ++i) asm volatile("" : "+v"(o.x[i][0]), "+v"(o.x[i][1]), "+v"(o.xe[i]));
    };
    // One stage's products; the next one's operands are read and a copy is begun in between.
    int buffer = 0;  // of the stage that is multiplied
    auto stage = [&](const Operands& now, Operands& next, int half) {
        // (behind the last stage an old one is read and copied again, for nothing)
        const int next_buffer = buffer + 1 == STAGES ? 0 : buffer + 1;
        const unsigned next_stage = next_buffer * STAGE;
        const int ahead = min(half + STAGES, halves - 1);
        const size_t on = offset_of(ahead);
        const uint32_t on_e = (uint32_t)(ahead >> 1) * e_step;
        constexpr int SLOTS = MI * NI - 1;
        bf16x8 wv[NI][4], xv[4];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < NI; ++j)
                values_of(__builtin_shufflevector(now.w[j][0], now.w[j][1], 0, 1, 2, 3, 4, 5, 6, 7), __uint_as_float((uint32_t)now.we[j] << 23), wv[j]);
        }
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const i32x8 x = __builtin_shufflevector(now.x[i][0], now.x[i][1], 0, 1, 2, 3, 4, 5, 6, 7);
            if constexpr (sizeof(T) == 4) values_of(x, __uint_as_float((uint32_t)now.xe[i] << 23), xv);
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const i32x8 w = __builtin_shufflevector(now.w[j][0], now.w[j][1], 0, 1, 2, 3, 4, 5, 6, 7);
                if constexpr (sizeof(T) == 2) {
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, acc[i][j], 0, 0, 0, now.we[j], 0, now.xe[i]);
                } else {
#pragma unroll
                    for (int h = 0; h < 4; ++h) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wv[j][h], xv[h], acc[i][j], 0, 0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
                const int t = i * NI + j;
                if (t == 0) {
                    // the next stage is there once no more than the ones behind it are on their way; then this one's buffer,
                    // which all waves have read, is filled again
                    wait_copies<(STAGES - 2) * COPIES>();
                    __builtin_amdgcn_s_barrier();
                } else {
                    // (early, so that they have arrived when the last product is through)
                    constexpr int READS = (NI + MI + SLOTS - 1) / SLOTS;
#pragma unroll
                    for (int k = (t - 1) * READS; k < t * READS && k < NI + MI; ++k) {
                        if (k < NI) read_w(next, next_stage, k);
                        else read_x(next, next_stage, k - NI);
                    }
#pragma unroll
                    for (int k = 0; k < COPIES; ++k)
                        if ((SLOTS >= COPIES + NI ? k + NI : k * SLOTS / COPIES) == t - 1) copy_one(buffer, on, on_e, k);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        landed(next);
        buffer = next_buffer;
    };
#pragma unroll
    for (int i = 0; i < STAGES; ++i) {
        const int half = min(i, halves - 1);
#pragma unroll
        for (int k = 0; k < COPIES; ++k) copy_one(i, offset_of(half), (uint32_t)(half >> 1) * e_step, k);
    }
    wait_copies<(STAGES - 1) * COPIES>();
    __builtin_amdgcn_s_barrier();
    Operands a, b;
#pragma unroll
    for (int j = 0; j < NI; ++j) read_w(a, 0, j);
#pragma unroll
    for (int i = 0; i < MI; ++i) read_x(a, 0, i);
    landed(a);
    for (int half = 0; half < halves; half += 2) {  // (an even number)
        stage(a, b, half);
        stage(b, a, half + 1);
    }
    wait_copies<0>();
    __builtin_amdgcn_s_barrier();  // (the stages' buffers are read no more)
    // Results go through LDS, 32 rows at a time, so that they are written in whole lines.
    constexpr int COLS = 32 * NI, PITCH = COLS + 4;  // floats
    float* mine = (float*)(lds + wave * (32 * PITCH * 4));
    const int col0 = (lane >> 5) * 4, cols = p.pair ? COLS / 2 : COLS, per_row = cols / 8, out0 = (tile0 + wn * 2 * NI) / (p.pair ? 2 : 1) * 16;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
#pragma unroll
        for (int j = 0; j < NI; ++j) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f32x4 v = {acc[i][j][4 * k], acc[i][j][4 * k + 1], acc[i][j][4 * k + 2], acc[i][j][4 * k + 3]};
                if (p.pair) {
                    if (k >= 2) continue;
#pragma unroll
                    for (int h = 0; h < 4; ++h) v[h] = silu<T>(v[h]) * acc[i][j][4 * (k + 2) + h];
                }
                *(f32x4*)(mine + row32 * PITCH + j * (p.pair ? 16 : 32) + k * 8 + col0) = v;
            }
        }
        const int row0 = (mt0 + (wm * MI + i) * 2) * 16;
        for (int e = lane; e < 32 * per_row; e += 64) {
            const int row = e / per_row, col = e % per_row * 8;
            const float* from_row = mine + row * PITCH + col;
            finish8<T>(p, row0 + row, out0 + col, *(const f32x4*)from_row, *(const f32x4*)(from_row + 4));
        }
    }
}

// An XCD takes whole panels of the weight, all rows of one after the other, so that a panel comes from memory once.  What its CUs have
// left over after whole rounds goes in tiles of half as many rows, if these are one round then (4096 rows by 22 016, 5.5 rounds for 6:
// 345 -> 340 us).  4096 rows by a pair of 11 008 x 4096: 335 us, 2.2 PFLOP/s, at which the chip lowers its clock; 1024 rows by
// 12 288 x 4096: 49 us, 2.1 PFLOP/s.
template <typename T, int MI, int NI>
__global__ __launch_bounds__(256, MI * NI <= 8 ? 2 : 1) void f8_tile_kernel(F8Product p, F8Shape s, F8Rows r, int m_groups, int n_groups) {
    constexpr bool HALVES = MI == 4 && NI > 2;
    __shared__ __attribute__((aligned(1024))) char lds[tile_lds(MI, NI)];
    const int xcd = blockIdx.x & 7, turn = blockIdx.x >> 3, all = (n_groups - xcd + 7) / 8 * m_groups;
    const int left = HALVES ? all % XCD_CUS : 0, whole = left <= XCD_CUS / 2 ? all - left : all;
    if (turn < whole) {
        f8_tile<T, MI, NI>(p, s, r, (turn / m_groups * 8 + xcd) * (4 * NI), turn % m_groups * (4 * MI), lds);
    } else if constexpr (HALVES) {
        const int t = whole + (turn - whole) / 2;
        if (t < all) {
            const int mt0 = t % m_groups * (4 * MI) + (turn - whole) % 2 * (2 * MI);
            if (mt0 * 16 < p.m) f8_tile<T, MI / 2, NI>(p, s, r, (t / m_groups * 8 + xcd) * (4 * NI), mt0, lds);
        }
    }
}

}  // namespace

// Up to 32 768 elements of sixteen rows at most are quantised by the workgroups that multiply them, which saves a launch of 3 us and the
// gap behind it, but is done by all of them (1 row by 4096 x 4096 6.4 us, apart 6.0 + 3.5; 16 rows by 12 288 x 4096 16.5, apart 11.3 + 2.9).
static bool quantised_first(int m, int steps) { return m > 16 || m * steps > 256; }

size_t f8_workspace(int m, int n, int k, int pair, int y_dtype) {
    const int steps = (k + 127) / 128;
    return quantised_first(m, steps) ? F8Rows{m, steps}.bytes() : 0;
}

hipError_t launch_f8_pack(const F8Shape& s, int dtype, const void* w, int64_t w_row, const void* up, int64_t up_row, char* weight, hipStream_t st) {
    const dim3 grid(s.steps(), (s.n + 127) / 128, s.pair ? 2 : 1);
    if (dtype == EE_BF16)
        EE_LAUNCH(f8_pack_kernel<__bf16>, grid, dim3(512), st, s, (const __bf16*)w, w_row, (const __bf16*)up, up_row, weight);
    else
        EE_LAUNCH(f8_pack_kernel<float>, grid, dim3(512), st, s, (const float*)w, w_row, (const float*)up, up_row, weight);
    return hipGetLastError();
}

hipError_t launch_f8_unpack(const F8Shape& s, int up, const char* weight, int dtype, void* w, hipStream_t st) {
    const dim3 grid((s.n + 15) / 16, s.steps());
    if (dtype == EE_BF16)
        EE_LAUNCH(f8_unpack_kernel<__bf16>, grid, dim3(64), st, s, up, weight, (__bf16*)w);
    else
        EE_LAUNCH(f8_unpack_kernel<float>, grid, dim3(64), st, s, up, weight, (float*)w);
    return hipGetLastError();
}

template <typename T, typename X, int MT, int NT, int W, int D>
static void launch_stream(const F8Product& p, const F8Shape& s, const F8Rows& r, hipStream_t st) {
    const int m_groups = ((p.m + 15) / 16 + MT - 1) / MT, n_groups = (s.tiles() + NT - 1) / NT;
    const size_t sums = (size_t)W * MT * NT * 1024, lds = __is_same(X, HeldRows) ? sums : std::max(sums, own_rows_bytes(p.m, s.steps()));
    EE_LAUNCH_SM((f8_stream_kernel<T, X, MT, NT, W, D>), dim3((n_groups + 7) / 8 * 8 * m_groups), dim3(W * 64), lds, st, p, s, r, m_groups, n_groups);
}

template <typename T, int MI, int NI>
static void launch_tile(const F8Product& p, const F8Shape& s, const F8Rows& r, hipStream_t st) {
    const int m_groups = (p.m + 64 * MI - 1) / (64 * MI), n_groups = (s.tiles() + 4 * NI - 1) / (4 * NI);
    const int most = (n_groups + 7) / 8 * m_groups;  // of an XCD; what is left over may be twice as many
    EE_LAUNCH((f8_tile_kernel<T, MI, NI>), dim3(8 * (most + (MI == 4 && NI > 2 ? XCD_CUS / 2 : 0))), dim3(256), st, p, s, r, m_groups, n_groups);
}

// What takes a product of more than 64 rows: the kind with the least time for a step of 128 elements, by the workgroups that it takes on
// 256 CUs; in ns, measured with bf16 results and weights that come from memory.  (fp32 results, whose steps take about twice as long in tiles,
// go by the same numbers.  A panel of the weight has one XCD: fewer than eight of them leave XCDs idle, which is not counted
// here: 4096 rows by 256 x 4096 take 32 us on four of them.)  Tiles run in rounds (alone: a workgroup that has its CU to
// itself, two: a pair that shares one), the others a few on a CU.  203 rows by 6656 x 6656: 8 x 4 tiles of 16 x 16 straight into registers 24 us,
// tiles of 128 x 128 through LDS 31; 256 rows by 12 288 x 4096: 32 and 25; 70 rows by 4096 x 4096: 4 x 2 9 us, 8 x 4 16.
struct Kind {
    int m, n;  // rows, rows of the weight, of a workgroup
    int alone, two;
};
static const Kind TILES[] = {{256, 256, 1720, 0}, {256, 192, 1540, 0}, {192, 192, 1200, 0}, {256, 128, 1140, 1980}, {128, 192, 1040, 1800}, {128, 128, 720, 1260}};
static const Kind STREAMS[] = {{128, 64, 500, 0}, {64, 64, 300, 0}, {64, 32, 250, 0}, {64, 16, 160, 0}};
constexpr int N_TILES = sizeof(TILES) / sizeof(Kind), N_STREAMS = sizeof(STREAMS) / sizeof(Kind);

static int kind_of(int m, int tiles, bool pair) {
    int best = 0;
    int64_t least = INT64_MAX;
    auto workgroups = [&](const Kind& k) { return (int64_t)((m + k.m - 1) / k.m) * ((tiles * 16 + k.n - 1) / k.n); };
    auto take = [&](int kind, int64_t t) {
        if (t < least) least = t, best = kind;
    };
    for (int i = 0; i < N_TILES; ++i) {
        const Kind& k = TILES[i];
        const int64_t n = workgroups(k), at_once = k.two ? 2 * CUS : CUS, left = n % at_once;
        const bool halves = k.m == 256 && !k.two;
        take(i, n / at_once * (k.two ? k.two : k.alone) + (left == 0 ? 0 : k.two && left > CUS ? k.two : halves && left <= CUS / 2 && n > CUS ? k.alone * 6 / 10 : k.alone));
    }
    for (int i = 0; i < N_STREAMS - (pair ? 1 : 0); ++i) {
        const Kind& k = STREAMS[i];
        const int64_t n = workgroups(k);
        take(N_TILES + i, i == 0 ? (n + CUS - 1) / CUS * k.alone : std::max<int64_t>(k.alone, n * (k.n * 30 / 8 + 70) / CUS));
    }
    return best;
}

// The launch of a product: one of the kinds above, or of what few rows take.
enum { OWN_2 = N_TILES + N_STREAMS, OWN_1, ROWS16_2, ROWS16_2_WIDE, ROWS16_1, ROWS32_1_WIDE, ROWS32_2, ROWS32_1 };
static int route_of(int m, int tiles, int steps, bool pair) {
    const int m_tiles = (m + 15) / 16;
    // (all widths of the framework's workloads, 1 row: within 0.4 us of the best of eight kinds)
    if (!quantised_first(m, steps)) return tiles >= 1024 || pair ? OWN_2 : OWN_1;
    // Few tiles: one to a workgroup, so that there are as many as CUs (16 rows by 4096 x 11 008: 11.3 us, two 15); many: two, four.
    // Up to 448 tiles, one each would leave many CUs a second workgroup (16 rows by 6656 x 6656, 416 tiles: two 10.6 us, one 12.0; by 7168 x 4096 8.0
    // and 8.4; by 7680 x 4096, 480 tiles, 9.0 and 8.6).
    if (m_tiles == 1) return pair || (tiles > 256 && tiles <= 448) ? ROWS16_2 : tiles >= 1024 ? ROWS16_2_WIDE : ROWS16_1;
    if (m_tiles == 2) return tiles <= 256 && !pair ? ROWS32_1_WIDE : ROWS32_2;
    if (m_tiles <= 4) {
        // as many workgroups as CUs, or a few more (64 rows by 2048 x 5504: two groups of rows 7.5 us, one 10.1; 61 rows by 4096 x 11 008, weights from
        // memory: one tile 18.7, two 21.6; 50 rows by 6656 x 6656: two 16.8, one 20.8)
        if (tiles <= 128 && !pair) return ROWS32_1;
        if (tiles <= 256 && !pair) return N_TILES + 3;
        return N_TILES + (tiles <= 512 ? 2 : 1);
    }
    return kind_of(m, tiles, pair);
}

template <typename T>
static void launch_product(const F8Product& p, const F8Shape& s, const F8Rows& r, hipStream_t st) {
    typedef HeldRows H;
    const bool bf16 = p.x_dtype == EE_BF16;
    switch (route_of(p.m, s.tiles(), s.steps(), p.pair)) {
        case 0: return launch_tile<T, 4, 4>(p, s, r, st);
        case 1: return launch_tile<T, 4, 3>(p, s, r, st);
        case 2: return launch_tile<T, 3, 3>(p, s, r, st);
        case 3: return launch_tile<T, 4, 2>(p, s, r, st);
        case 4: return launch_tile<T, 2, 3>(p, s, r, st);
        case 5: return launch_tile<T, 2, 2>(p, s, r, st);
        case 6: return launch_stream<T, H, 8, 4, 4, 2>(p, s, r, st);
        case 7: return launch_stream<T, H, 4, 4, 4, 2>(p, s, r, st);
        case 8: return launch_stream<T, H, 4, 2, 4, 2>(p, s, r, st);
        case 9: return launch_stream<T, H, 4, 1, 4, 4>(p, s, r, st);
        case OWN_2: return bf16 ? launch_stream<T, __bf16, 1, 2, 8, 2>(p, s, r, st) : launch_stream<T, float, 1, 2, 8, 2>(p, s, r, st);
        case OWN_1: return bf16 ? launch_stream<T, __bf16, 1, 1, 8, 2>(p, s, r, st) : launch_stream<T, float, 1, 1, 8, 2>(p, s, r, st);
        case ROWS16_2: return launch_stream<T, H, 1, 2, 4, 4>(p, s, r, st);
        case ROWS16_2_WIDE: return launch_stream<T, H, 1, 2, 8, 2>(p, s, r, st);
        case ROWS16_1: return launch_stream<T, H, 1, 1, 4, 4>(p, s, r, st);
        case ROWS32_1_WIDE: return launch_stream<T, H, 2, 1, 8, 2>(p, s, r, st);
        case ROWS32_2: return launch_stream<T, H, 2, 2, 4, 4>(p, s, r, st);
        default: return launch_stream<T, H, 2, 1, 4, 4>(p, s, r, st);  // ROWS32_1
    }
}

void f8_launch_shape(int m, int n, int k, int pair, int32_t shape[4]) {
    static const int FEW[][3] = {{16, 32, 8}, {16, 16, 8}, {16, 32, 4}, {16, 32, 8}, {16, 16, 4}, {32, 16, 8}, {32, 32, 4}, {32, 16, 4}};
    const F8Shape s{n, k, pair};
    const int kind = route_of(m, s.tiles(), s.steps(), pair);
    const Kind& many = kind < N_TILES ? TILES[kind] : STREAMS[std::min(kind - N_TILES, N_STREAMS - 1)];
    const bool few = kind >= N_TILES + N_STREAMS;
    shape[0] = few ? FEW[kind - OWN_2][0] : many.m;
    shape[1] = few ? FEW[kind - OWN_2][1] : many.n;
    shape[2] = few ? FEW[kind - OWN_2][2] : 4;
    shape[3] = kind < N_TILES ? 2 : kind == OWN_1 || kind == OWN_2 ? 1 : 0;
}

hipError_t launch_f8_matmul(const F8Product& p, hipStream_t st) {
    const F8Shape s{p.n, p.k, p.pair};
    const F8Rows r{p.m, s.steps()};
    if (quantised_first(p.m, s.steps())) {
        const dim3 rows_grid((p.m + 15) / 16, (r.steps + 3) / 4);
        if (p.x_dtype == EE_BF16)
            EE_LAUNCH(f8_rows_kernel<__bf16>, rows_grid, dim3(256), st, r, (const __bf16*)p.x, p.x_row, p.k, p.workspace);
        else
            EE_LAUNCH(f8_rows_kernel<float>, rows_grid, dim3(256), st, r, (const float*)p.x, p.x_row, p.k, p.workspace);
    }
    if (p.y_dtype == EE_BF16)
        launch_product<__bf16>(p, s, r, st);
    else
        launch_product<float>(p, s, r, st);
    return hipGetLastError();
}

}  // namespace ee
