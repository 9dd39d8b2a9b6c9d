// xred_product_choice.hpp -- which kernel takes a product, by types, sizes and alignment.
//
// Results have the same bits whatever the alignment, the distance between rows and the part
// of the chip that the device is: all kernels add in the same order, but for the streaming
// ones, which sum each half of the steps by itself, and those are chosen by types and sizes alone.
#pragma once

#include "xred_product_narrow.hpp"

namespace xred {

// Tiles of 256 x 256 fill the chip from about half a tile a CU on, even if few of their rows
// exist (64 experts, 2048 x 2048: 8192 rows 165 us, tiles of 128 x 128 189, mx4 78 and 92;
// 4096 rows 165 and 161, mx4 70 and 69; the gradient of as many 170 and 266).  fp32, whose
// matrix instructions take eight times as long, keeps smaller tiles as busy and loses more by
// rows that do not exist: 32768 rows of 4096 x 1024 2130 and 2390, but 8192 of 2048 x 2048
// 1133 and 895 and the gradient of 32768 2630 and 2380.
inline bool wide_pays(const ProductParams &p, bool grad, bool f32)
{
    const uint64_t columns = (p.n + 255) / 256;
    const uint64_t rows = grad ? (uint64_t)p.experts * ((p.m + 255) / 256)
                               : p.rows / 256 + (p.rows < p.experts ? p.rows : p.experts);
    if (f32 && (grad || p.rows < 256ull * p.experts || rows * columns < 1024)) return false;
    return p.n > 128 && rows * columns >= 128;
}

// Few rows for an expert: its weights are what costs (64 experts, bf16: 8 rows of 4096 x 4096
// 47 us, 71 in 128 x 128 tiles; 2048 rows of 2048 x 4096 209, in wide tiles 187).  And where
// larger tiles would leave CUs without one, more of them with more steps on their way (one
// expert, 220 rows of 299 x 2045: 14.7 us, in 64 x 64 tiles 23.8; 2048 x 4096 18.5 and 24.8;
// 64 experts, 2048 rows of 299 x 2045 23 and 38; from 64 x 64 tiles for every CU on it turns:
// 8 experts, 2000 rows of 640 x 320 7.8 and 6.2).  At 64 elements and more, which pieces and
// mx4's exponents are read in whole.
//
// The host knows the rows that x has, not those that exist or which expert has them.  64 experts
// of 4096 x 2048 bf16, in a buffer of 32768 rows (wide tiles) and in one of their own size: 4096
// rows 250 and 203 us, 512 rows 232 and 181, 64 rows 119 and 110.  256 experts of 2048 x 2048,
// 4096 rows, narrow tiles: 374 us with 16 rows each, 425 with 3841 of them in one expert.
constexpr uint64_t kChipCus = 256;   // of the whole chip, even if the device is a part of it
inline bool narrow_pays(const ProductParams &p)
{
    if (p.n < 64 || p.k < 64) return false;
    const uint64_t tiles = (p.rows / 64 + (p.rows < p.experts ? p.rows : p.experts)) * (uint64_t)((p.n + 63) / 64);
    return p.rows <= 16ull * p.experts || tiles <= kChipCus ||
           (p.rows <= 32ull * p.experts && tiles < 2 * kChipCus);
}

// Rows 8 MB and more apart are past the streaming tiles' 32-bit offsets.
template <class P, bool ACROSS, bool DIRECT>
hipError_t go_few(const ProductParams &p, hipStream_t s)
{
    return p.row_stride < kWideStride && p.col_stride < kWideStride
               ? go_narrow<P, ACROSS, DIRECT>(p, s)
               : go_product<P, false, ACROSS, DIRECT, 1, 1, true>(p, s);
}

// Tiles of 64 x 64 where there are too few of 128 x 128 to keep the chip busy, and in fp32,
// bound by its matrix instructions, where experts would leave most of 128 rows empty (64
// experts, 4096 rows of 2048 x 2048: 526 us, 643 in 128 x 128 tiles).
template <class P, bool GRAD, bool ACROSS, bool DIRECT>
hipError_t go_tiles(const ProductParams &p, hipStream_t s)
{
    const uint64_t rows = GRAD ? (uint64_t)p.experts * ((p.m + 127) / 128)
                               : p.rows / 128 + (p.rows < p.experts ? p.rows : p.experts);
    const bool small = (P::kSize == 4 && !GRAD && p.rows < 96ull * p.experts) ||
                       rows * ((p.n + 127) / 128) < 2 * device_cus();
    return small ? go_product<P, GRAD, ACROSS, DIRECT, 1, 1>(p, s)
                 : go_product<P, GRAD, ACROSS, DIRECT, 2, 2>(p, s);
}

template <class P>
hipError_t launch_product_plain(const ProductParams &p, bool grad, bool across, hipStream_t s)
{
    constexpr uint64_t es = P::kSize;
    const bool direct = grad ? on_grid(p.row, p.row_stride, 0, p.m * es) &&
                                   on_grid(p.col, p.col_stride, 0, p.n * es)
                             : on_grid(p.row, p.row_stride, 0, p.k * es) &&
                                   on_grid(p.col, p.col_stride, p.col_expert, (across ? p.n : p.k) * es);
    if (!grad && narrow_pays(p)) {
        if (across)
            return direct ? go_few<P, true, true>(p, s) : go_few<P, true, false>(p, s);
        return direct ? go_few<P, false, true>(p, s) : go_few<P, false, false>(p, s);
    }
    if (p.row_stride < kWideStride && p.col_stride < kWideStride && wide_pays(p, grad, es == 4)) {
        using O = typename OwnType<P>::T;
        if (direct)
            return p.out_type == XRED_FLOAT32 ? launch_wide<P, TF32>(p, grad, across, s)
                                              : launch_wide<P, O>(p, grad, across, s);
        // Loose operands, 64 experts, bf16: 32768 rows of 4097 x 2049 1343 us, tiles of
        // 128 x 128 2160 (transposed 1090 and 2090); 8192 rows of 2049 x 2047 310 and 294,
        // 4096 rows 300 and 229.
        if (!grad && p.out_type == dtype_of<O>() && p.rows >= 192ull * p.experts)
            return across ? go_wide<P, O, false, true, false, false>(p, s)
                          : go_wide<P, O, false, false, false, false>(p, s);
    }
    if (grad)
        return direct ? go_tiles<P, true, true, true>(p, s) : go_tiles<P, true, true, false>(p, s);
    if (across)
        return direct ? go_tiles<P, false, true, true>(p, s) : go_tiles<P, false, true, false>(p, s);
    return direct ? go_tiles<P, false, false, true>(p, s) : go_tiles<P, false, false, false>(p, s);
}

// Whether scales can be read by whole words (mx4: its exponents, four of them).
template <class P>
inline bool scale_words(const ProductParams &p)
{
    return (__is_same(P, PE4M3) ||
            ((uintptr_t)p.row_scale | p.row_scale_stride | (uintptr_t)p.col_scale | p.col_scale_stride |
             p.col_scale_expert | p.k / 16) % 4 == 0) &&
           p.row_scale_stride < kWideStride && p.col_scale_stride < kWideStride;
}

template <class P>
hipError_t launch_product_scaled(const ProductParams &p, hipStream_t s)
{
    const bool direct = on_grid(p.row, p.row_stride, 0, p.k) &&
                        on_grid(p.col, p.col_stride, p.col_expert, p.k);
    if (narrow_pays(p))
        return direct ? go_few<P, false, true>(p, s) : go_few<P, false, false>(p, s);
    if (direct && p.row_stride < kWideStride && p.col_stride < kWideStride && scale_words<P>(p) &&
        wide_pays(p, false, false))
        return p.out_type == XRED_FLOAT32    ? launch_wide<P, TF32>(p, false, false, s)
               : p.out_type == XRED_BFLOAT16 ? launch_wide<P, TBF16>(p, false, false, s)
                                             : launch_wide<P, TF16>(p, false, false, s);
    return direct ? go_tiles<P, false, false, true>(p, s) : go_tiles<P, false, false, false>(p, s);
}

}  // namespace xred
