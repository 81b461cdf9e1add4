// Products with weights held in 8 bits (ee_f8_* of ee.h): layout of a packed weight and of quantised rows, and the launches.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "ee.h"

namespace ee {

// 16 rows (of a weight, or of x) by 128 elements of the contraction are one fragment of 2048 bytes, in the order in which a wave's
// lanes hold an operand of the 8-bit matrix instructions: two halves of 16 bytes per lane, so that every load is one contiguous
// kilobyte.  Lane = 16 * quarter + row holds elements 32 * quarter .. + 31, the first 16 in half 0.  A weight is
// [n tiles][k steps] fragments and, behind them, [k steps][n tiles, rounded up to 4] bytes of exponents (e + 127); of a pair, tile 2i is the gate's tile i and tile 2i + 1 the
// up weight's, so that a wave that has both multiplies them where they are.  Quantised rows are [m tiles][k steps] fragments and
// [m tiles][k steps][16] exponents.  What lies behind n, m and k is zero.
constexpr int F8_FRAGMENT = 2048;

struct F8Shape {
    int n, k, pair;
    constexpr int tiles() const { return (n + 15) / 16 * (pair ? 2 : 1); }
    constexpr int steps() const { return (k + 127) / 128; }
    constexpr size_t exponents() const { return (size_t)tiles() * steps() * F8_FRAGMENT; }  // where they begin
    constexpr int exponent_row() const { return (tiles() + 3) / 4 * 4; }
    constexpr size_t bytes() const { return exponents() + (size_t)exponent_row() * steps(); }
};

struct F8Rows {
    int m, steps;
    constexpr size_t exponents() const { return (size_t)((m + 15) / 16) * steps * F8_FRAGMENT; }
    constexpr size_t bytes() const { return exponents() + ((size_t)((m + 15) / 16) * steps * 16 + 255) / 256 * 256; }
};

struct F8Product {
    int m, n, k, pair;
    const char* weight;
    const void* x;
    int x_dtype;
    int64_t x_row;
    void* y;
    int y_dtype;
    int64_t y_row;
    const void* add;
    int64_t add_row;
    char* workspace;
};

void f8_launch_shape(int m, int n, int k, int pair, int32_t shape[4]);
size_t f8_workspace(int m, int n, int k, int pair, int y_dtype);
hipError_t launch_f8_pack(const F8Shape& s, int dtype, const void* w, int64_t w_row, const void* up, int64_t up_row, char* weight, hipStream_t st);
hipError_t launch_f8_unpack(const F8Shape& s, int up, const char* weight, int dtype, void* w, hipStream_t st);
hipError_t launch_f8_matmul(const F8Product& p, hipStream_t st);

}  // namespace ee
