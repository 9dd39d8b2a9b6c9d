// xred_product_narrow.hpp -- the experts' products of few rows each, a decode batch, and of
// too few tiles to fill the chip with larger ones.
//
// Bound by HBM: the weights of every expert that has rows are read once (from L2 again for
// every 32 rows more), and all that counts is to keep enough of them on their way.  A tile is
// 32 rows by 64 columns; four steps of k lie in LDS (48 KB, so that three workgroups share a
// CU), three of them on their way at any time, and go on from a tile into the next one without
// a pause.  Two waves have a block of 32 columns each for one half of every step, two for the
// other half; the halves meet in LDS at the tile's end.
//
// 8 rows of 64 experts, 4096 x 4096: bf16 50 us, 5.4 TB/s (128 x 128 tiles, one step on its
// way: 71), transposed 65 (100), e4m3 32 (33), mx4 17 (31), 4097 x 4099 bf16 98 (116).  488
// rows of 128 experts, of which 86 have some, mx4: 168 us, 4.7 TB/s (280).
#pragma once

#include "xred_product_wide.hpp"

namespace xred {

// GRID: operands on the 16-byte grid, in whole pieces; others are on their way in registers.
template <class P, bool ACROSS, bool GRID>
__global__ __launch_bounds__(kProductThreads, 3) void product_narrow_kernel(ProductParams p)
{
    constexpr int BM = 32, BN = 64;
    constexpr bool kMx4 = __is_same(P, PMx4), kE4M3 = __is_same(P, PE4M3), kScaled = kMx4 || kE4M3;
    using Rows = std::conditional_t<GRID, WideOperand<P, false, BM>, LooseOperand<P, false, BM, uint32_t>>;
    using Columns = std::conditional_t<GRID, WideOperand<P, ACROSS, BN>, LooseOperand<P, ACROSS, BN, uint32_t>>;
    // an array for each step: a read of one does not wait for loads into another
    __shared__ __attribute__((aligned(1024))) char rows0[4096], rows1[4096], rows2[4096], rows3[4096];
    __shared__ __attribute__((aligned(1024))) char columns0[8192], columns1[8192], columns2[8192], columns3[8192];
    __shared__ uint32_t first[XRED_MAX_EXPERTS], shared[kProductThreads / 64];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t wc = wave % 2, part = wave / 2;   // this wave's columns and half of a step
    const uint32_t l = threadIdx.x % 64, h = l / 32;
    RowTiles<kProductThreads> all;
    all.start(p, shared, [&](uint32_t n) { return (n + BM - 1) / BM * p.col_tiles; });
#pragma unroll
    for (int j = 0; j < RowTiles<kProductThreads>::kEach; ++j)
        first[threadIdx.x * RowTiles<kProductThreads>::kEach + j] = all.first[j];
    const uint32_t total = __builtin_amdgcn_readfirstlane(all.total);
    __syncthreads();

    uint32_t place = blockIdx.x;
    auto next = [&](WideTile &w) {
        uint32_t i, lo, hi, tiles;
        for (;; place += gridDim.x) {
            if (place / 8 >= (total + 7) / 8) return false;
            if (!tile_of(place, total, i)) continue;
            uint32_t upto = 0;   // experts whose first tile is i or before
            for (uint32_t e = 0; e < p.experts; e += 64)
                upto += __popcll(__builtin_amdgcn_ballot_w64(e + l < p.experts && first[e + l] <= i));
            if (upto == 0) continue;
            w.expert = __builtin_amdgcn_readfirstlane(upto - 1);
            i -= __builtin_amdgcn_readfirstlane(first[w.expert]);
            uniform_rows(p, w.expert, lo, hi);
            tiles = (hi - lo + BM - 1) / BM;   // side by side: the same weights
            // else offsets do not ascend, and the sum has overflowed
            if (i < tiles * p.col_tiles) break;
        }
        place += gridDim.x;
        w.row = lo + i % tiles * BM;
        w.rows = hi - w.row;
        w.column = i / tiles * BN;
        return true;
    };

    const uint32_t length = p.k * P::kSize, along = ACROSS ? p.k : length;
    const uint32_t steps = (length + 127) / 128, groups = (steps + 3) / 4;
    const uint32_t count = kMx4 ? p.k / 16 : steps * 4;   // bytes of a row's scales
    Rows rows;
    Columns columns;
    const char *row_scale = nullptr, *column_scale = nullptr;   // this lane's
    bool more;
    auto begin = [&](const WideTile &w) {
        const uint32_t tid = threadIdx.x;
        rows.start(p.row + w.row * p.row_stride, p.row_stride, w.rows, length, tid);
        columns.start(p.col + w.expert * p.col_expert +
                          w.column * (ACROSS ? (uint64_t)P::kSize : p.col_stride),
                      p.col_stride, p.n - w.column, along, tid);
        if constexpr (kScaled) {
            const uint32_t left = w.rows < BM ? w.rows : BM, row = l % 32 < left ? l % 32 : left - 1;
            uint32_t column = w.column + wc * 32 + (kMx4 ? l % 32 : 0);
            column = (column < p.n ? column : p.n - 1) / (kE4M3 ? 128 : 1);
            row_scale = p.row_scale + (w.row + row) * p.row_scale_stride;
            column_scale = p.col_scale + w.expert * p.col_scale_expert + column * p.col_scale_stride;
        }
    };
    // mx4: the four exponents of this lane's half of step t, or where its row's last four are
    auto scale_place = [&](uint32_t t) {
        const uint32_t at = kMx4 ? t * 8 + 4 * h : t * 4;
        return at < count - 4 ? at : count - 4;
    };
    uint32_t rs[4], cs[4];   // scales on their way, for each step in LDS
    u32x4 row_held[4][GRID ? 1 : Rows::kPieces], column_held[4][GRID ? 1 : Columns::kPieces];
    // Step t, which is past the last (of k, or of all tiles) where nothing is loaded: the same
    // number of loads, so that waits can count them.
    auto load = [&](auto stage, uint32_t t, lds_bytes to_rows, lds_bytes to_columns) {
        constexpr int J = decltype(stage)::value;
        const bool there = more && t < steps;
        if constexpr (kScaled) {
            const uint32_t at = scale_place(t);
            rs[J] = *(const __attribute__((address_space(1))) u32_any *)((global_bytes)row_scale + at);
            cs[J] = *(const __attribute__((address_space(1))) u32_any *)((global_bytes)column_scale + at);
        }
        if constexpr (GRID) {
            rows.load_if(there, t, length, to_rows);
            columns.load_if(there, t, along, to_columns);
        } else {
            rows.fetch_any(there ? t : 0, row_held[J]);
            columns.fetch_any(there ? t : 0, column_held[J]);
        }
    };
    constexpr int kLoads = 3 + (kScaled ? 2 : 0);
    f32x16 acc = f32x16{};
    auto multiply_step = [&](auto stage, uint32_t t, lds_bytes from_rows, lds_bytes from_columns) {
        constexpr int J = decltype(stage)::value;
        u32x4 rf[2], cf[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            rf[s] = Rows::fragment(from_rows, 0, part * 2 + s, l);
            cf[s] = Columns::fragment(from_columns, wc, part * 2 + s, l);
        }
        if constexpr (kE4M3) {
            const f32x16 sums = multiply_e4m3(cf[0], cf[1], rf[0], rf[1], f32x16{});
            const float by = __uint_as_float(rs[J]) * __uint_as_float(cs[J]);
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[j] = __builtin_fmaf(sums[j], by, acc[j]);
        } else if constexpr (kMx4) {
            const uint32_t at = t * 8 + 4 * h, skip = (at - scale_place(t)) * 8 + part * 16;
            const uint32_t re = skip < 32 ? rs[J] >> skip : 0, ce = skip < 32 ? cs[J] >> skip : 0;
            acc = multiply_mx4<0>(cf[0], rf[0], ce, re, acc);
            acc = multiply_mx4<1>(cf[1], rf[1], ce, re, acc);
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s) acc = multiply<P>(cf[s], rf[s], acc);
        }
    };

    const lds_bytes r[4] = {(lds_bytes)rows0, (lds_bytes)rows1, (lds_bytes)rows2, (lds_bytes)rows3};
    const lds_bytes c[4] = {(lds_bytes)columns0, (lds_bytes)columns1, (lds_bytes)columns2, (lds_bytes)columns3};
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I3 = std::integral_constant<int, 3>;
    WideTile w, ahead;
    more = next(w);
    if (!more) return;
    begin(w);
    ahead = w;
    load(I0{}, 0, r[0], c[0]);
    load(I1{}, 1, r[1], c[1]);
    load(I2{}, 2, r[2], c[2]);
    // loose: the tile's whose steps go to LDS; loads may be in the next one's already
    Rows put_rows;
    Columns put_columns;
    // the step that this wave's loads of two later ones follow is there, for all waves after
    // the barrier, and what the step before it lay in is free
    auto turn = [&](auto stage, uint32_t t) {
        constexpr int J = decltype(stage)::value;
        if constexpr (!GRID) {
            if (Columns::is_whole(t, along) && Rows::is_whole(t, length)) {
                put_rows.template put<true>(t, length, r[J], row_held[J]);
                put_columns.template put<true>(t, along, c[J], column_held[J]);
            } else {
                put_rows.template put<false>(t, length, r[J], row_held[J]);
                put_columns.template put<false>(t, along, c[J], column_held[J]);
            }
            __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        } else if constexpr (kLoads == 5) __asm__ volatile("s_waitcnt vmcnt(10) lgkmcnt(0)" ::: "memory");
        else __asm__ volatile("s_waitcnt vmcnt(6) lgkmcnt(0)" ::: "memory");
        static_assert(kLoads == 5 || kLoads == 3, "the counts above");
        __builtin_amdgcn_s_barrier();
        __asm__ volatile("" ::: "memory");
    };
    for (;;) {
        acc = f32x16{};
        put_rows = rows;
        put_columns = columns;
        bool last;
        for (uint32_t g = 0; g < groups; ++g) {
            const uint32_t t = g * 4;
            last = g + 1 == groups;
            turn(I0{}, t);
            load(I3{}, t + 3, r[3], c[3]);
            multiply_step(I0{}, t, r[0], c[0]);
            turn(I1{}, t + 1);
            if (last) {   // on into the next tile
                more = next(ahead);
                if (more) begin(ahead);
            }
            const uint32_t u = last ? 0 : t + 4;
            load(I0{}, u, r[0], c[0]);
            if (t + 1 < steps) multiply_step(I1{}, t + 1, r[1], c[1]);
            turn(I2{}, t + 2);
            load(I1{}, u + 1, r[1], c[1]);
            if (t + 2 < steps) multiply_step(I2{}, t + 2, r[2], c[2]);
            turn(I3{}, t + 3);
            load(I2{}, u + 2, r[2], c[2]);
            if (t + 3 < steps) multiply_step(I3{}, t + 3, r[3], c[3]);
        }
        // the last step's place is free until the next is loaded there
        __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        const lds_bytes mine = c[3] + wc * 4096 + l * 16;
        if (part == 1) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(__attribute__((address_space(3))) u32x4 *)(mine + q * 1024) =
                    u32x4{__float_as_uint(acc[4 * q]), __float_as_uint(acc[4 * q + 1]),
                          __float_as_uint(acc[4 * q + 2]), __float_as_uint(acc[4 * q + 3])};
        }
        __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        __asm__ volatile("" ::: "memory");
        if (part == 0) {
            char *to = p.out + (w.row + l % 32) * p.out_stride;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const u32x4 other = *(const __attribute__((address_space(3))) u32x4 *)(mine + q * 1024);
                const uint32_t col = w.column + wc * 32 + 8 * q + 4 * h;
                if (l % 32 >= w.rows || col >= p.n) continue;
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = acc[4 * q + j] + __uint_as_float(other[j]);
                store_four(to, col, p.n - col < 4 ? p.n - col : 4, v, p.out_type);
            }
        }
        if (!more) break;
        w = ahead;
    }
}

template <class P, bool ACROSS, bool GRID>
hipError_t go_narrow(ProductParams p, hipStream_t s)
{
    p.col_tiles = (p.n + 63) / 64;
    const uint64_t tiles = (p.rows / 32 + (p.rows < p.experts ? p.rows : p.experts)) * (uint64_t)p.col_tiles;
    p.most = (uint32_t)tiles;
    const uint64_t most = 3 * device_cus();   // at once
    return launch_kernel(product_narrow_kernel<P, ACROSS, GRID>,
                         dim3(grid_of(tiles < most ? (tiles + 7) / 8 * 8 : most, kProductThreads)),
                         dim3(kProductThreads), 0, s, p);
}

}  // namespace xred
