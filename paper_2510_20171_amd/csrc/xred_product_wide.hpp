// xred_product_wide.hpp -- the experts' products in tiles of 256 x 256, for calls with
// enough rows to fill the chip with them.
//
// A workgroup of four waves has a CU to itself: each wave keeps 128 x 128 sums in its
// 256 accumulation registers, so that a fragment of either operand is used four times
// and LDS is read at half of its rate while the matrix cores run.  Two steps of k (128
// KB) are in LDS, one being multiplied, the next on its way by loads straight to LDS; a
// step's buffer is free once its last fragments are read, three quarters through it, and
// is filled again at once.  Fragments are read one sub-step ahead, one between every two
// matrix instructions.
//
// Buffer descriptors bound every load: what lies past the operand's rows, columns or k
// comes as zero, so ragged tiles run the same code.  A tile of at most 128 or 64 rows
// has a main loop of its own that does a half or a quarter of the products.
//
// Workgroups stay for several tiles.  The first two steps of the next tile are loaded
// before the results of the last one go out, through LDS (32 KB beside the operands'), in
// whole 128-byte pieces of rows.
#pragma once

#include "xred_product.hpp"

namespace xred {

constexpr uint32_t kOutside = 0x80000000u;   // an offset past every descriptor's range
constexpr uint64_t kWideStride = 1u << 23;   // bytes between rows are below this

// M matrix instructions with R reads of LDS, L loads and W writes to LDS spread among
// them.
template <int R, int M, int L, int W, int J = 0>
__device__ __forceinline__ void interleave()
{
    if constexpr (J < M) {
        constexpr int r = R * (J + 1) / M - R * J / M, l = L * (J + 1) / M - L * J / M;
        constexpr int w = W * (J + 1) / M - W * J / M;
        if constexpr (r > 0) __builtin_amdgcn_sched_group_barrier(0x100, r, 0);
        if constexpr (l > 0) __builtin_amdgcn_sched_group_barrier(0x20, l, 0);
        if constexpr (w > 0) __builtin_amdgcn_sched_group_barrier(0x200, w, 0);
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        interleave<R, M, L, W, J + 1>();
    }
}

// 256 rows (along) or columns (across) of an operand, a tile's.
template <class P, bool ACROSS>
struct WideOperand {
    static constexpr int kPieces = 8;                  // of a thread and step
    static constexpr int kWide = 256 * P::kSize / 16;  // across: pieces of a row of k
    static constexpr int kRows = 128 / P::kSize;       // across: rows of k in a step
    static constexpr int kReads = ACROSS ? (P::kSize == 2 ? 2 : 4) : 1;   // of a fragment

    const char *base;      // the same in every lane
    uint64_t step, bytes;  // from one step to the next; from base to the operand's end
    uint32_t at[kPieces];
    u32x4 held[kPieces];   // of a step on its way through registers

    // items: rows or columns that exist; length: of k, in bytes (along) or rows (across).
    __device__ __forceinline__ void start(const char *from, uint64_t stride, uint32_t items,
                                          uint32_t length, uint32_t tid)
    {
        base = from;
        step = ACROSS ? stride * kRows : 128;
        bytes = ACROSS ? (length - 1) * stride + (uint64_t)items * P::kSize
                       : (uint64_t)(items < 256 ? items - 1 : 255) * stride + length;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint32_t q = (tid / 64 * kPieces + i) * 64 + tid % 64;
            if constexpr (ACROSS) {
                const uint32_t row = q / kWide;
                uint32_t piece = q % kWide;
                if constexpr (P::kSize == 2) piece ^= (row % 4) * 2;
                at[i] = piece * 16 < items * P::kSize ? row * (uint32_t)stride + piece * 16 : kOutside;
            } else {
                const uint32_t row = q / 8, piece = q % 8 ^ row % 8;
                at[i] = row < items ? row * (uint32_t)stride + piece * 16 : kOutside;
            }
        }
    }

    __device__ __forceinline__ rsrc_t range(uint32_t t) const
    {
        const uint64_t left = bytes - t * step;
        return make_rsrc(base + t * step, left < kOutside ? (uint32_t)left : kOutside);
    }
    // Where piece i of step t is.  WHOLE: k goes on past the step.
    template <bool WHOLE>
    __device__ __forceinline__ uint32_t offset(int i, uint32_t t, uint32_t length) const
    {
        if constexpr (ACROSS || WHOLE) return at[i];
        // the end of a row is not the end of the operand
        const uint32_t q = (threadIdx.x / 64 * kPieces + i) * 64 + threadIdx.x % 64;
        return (q % 8 ^ q / 8 % 8) * 16 < length - t * 128 ? at[i] : kOutside;
    }

    // Step t straight into LDS.
    template <bool WHOLE>
    __device__ __forceinline__ void load(uint32_t t, uint32_t length, lds_bytes to) const
    {
        const rsrc_t r = range(t);
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                r, (__attribute__((address_space(3))) void *)(to + (wave * kPieces + i) * 1024), 16,
                (int)offset<WHOLE>(i, t, length), 0, 0, 0);
    }

    // The same by way of registers: fetch(), and later put().
    template <bool WHOLE>
    __device__ __forceinline__ void fetch(uint32_t t, uint32_t length)
    {
        const rsrc_t r = range(t);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) held[i] = bload<kLoadKeep>(r, offset<WHOLE>(i, t, length));
    }
    __device__ __forceinline__ void put(lds_bytes to) const
    {
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            *(__attribute__((address_space(3))) u32x4 *)(
                to + ((threadIdx.x / 64 * kPieces + i) * 64 + threadIdx.x % 64) * 16) = held[i];
    }

    static __device__ __forceinline__ u32x4 fragment(lds_bytes from, int b, int s, uint32_t lane)
    {
        return Operand<P, ACROSS, true, 256>::fragment(from, b, s, lane);
    }
};

// The thread's number, anew: what is computed from it is not kept in registers from one
// tile to the next.
__device__ __forceinline__ uint32_t fresh_thread()
{
    uint32_t t = threadIdx.x;
    __asm__ volatile("" : "+v"(t));
    return t;
}

// A tile, the same in every lane.
struct WideTile {
    uint32_t expert, row, rows, column;   // first row of x (gradient: of dw), rows that exist
    uint32_t length, steps;               // of k: bytes (gradient: rows); steps
    uint32_t first;                       // gradient: the expert's first row
};

// Rows of expert e, known to be the same in every lane.
__device__ __forceinline__ void uniform_rows(const ProductParams &p, uint32_t e, uint32_t &lo, uint32_t &hi)
{
    expert_rows(p, e, lo, hi);
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
}

// O: the output's type.  ADD: onto what it holds (gradient).
template <class P, class O, bool GRAD, bool ACROSS, bool ADD>
__global__ __launch_bounds__(kProductThreads, 1) void product_wide_kernel(ProductParams p)
{
    using Rows = WideOperand<P, GRAD>;
    using Columns = WideOperand<P, ACROSS>;
    constexpr bool kMx4 = __is_same(P, PMx4);
    __shared__ __attribute__((aligned(1024))) char rows0[32768], rows1[32768];
    __shared__ __attribute__((aligned(1024))) char columns0[32768], columns1[32768];
    constexpr int kStage = 32 * 144;   // results of a wave on their way out
    __shared__ __attribute__((aligned(16))) char stage[4 * kStage];
    __shared__ uint32_t first[GRAD ? 1 : XRED_MAX_EXPERTS];   // tile of each expert
    __shared__ uint32_t shared[4];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t wr = wave / 2, wc = wave % 2;
    // Work comes in items: a tile, or (p.spans) as many columns' tiles of an expert's last
    // rows as take about as long, two or three if those rows are at most 128 or 64.
    auto span = [&](uint32_t rest) { return p.spans ? rest > 64 ? 2u : 3u : 1u; };
    auto whole_tiles = [](uint32_t n) { return n / 256 + (n % 256 > 128); };
    uint32_t total;   // items
    // gradient: an expert's tiles are dealt to all XCDs where there are enough of them,
    // since experts' rows, and with them the tiles' lengths, differ
    const uint32_t of_expert = p.row_tiles * p.col_tiles, share = of_expert < 64 ? 0 : (of_expert + 7) / 8;
    if constexpr (GRAD) {
        total = share ? p.experts * share * 8 : p.experts * of_expert;
    } else {
        RowTiles<kProductThreads> all;
        all.start(p, shared, [&](uint32_t n) {
            const uint32_t rest = n % 256, s = span(rest);
            return whole_tiles(n) * p.col_tiles +
                   (rest == 0 || rest > 128 ? 0 : (p.col_tiles + s - 1) / s);
        });
#pragma unroll
        for (int j = 0; j < RowTiles<kProductThreads>::kEach; ++j)
            first[threadIdx.x * RowTiles<kProductThreads>::kEach + j] = all.first[j];
        total = __builtin_amdgcn_readfirstlane(all.total);
        __syncthreads();
    }
    // Tile i of `rows` x `columns` of them: groups of four rows, column by column.
    auto grouped = [](uint32_t i, uint32_t rows, uint32_t columns, uint32_t &row, uint32_t &column) {
        const uint32_t group = i / (4 * columns), rest = i - group * 4 * columns;
        const uint32_t left = rows - group * 4, high = left < 4 ? left : 4;
        row = group * 4 + rest % high;
        column = rest / high;
    };
    uint32_t place = blockIdx.x, columns_left = 0;
    // the next of this workgroup's tiles, w being the last; false: none is left
    auto next = [&](WideTile &w) {
        if (columns_left) {
            --columns_left;
            w.column += 256;
            return true;
        }
        if constexpr (GRAD) {
            uint32_t i;
            for (;; place += gridDim.x) {
                if (place >= total) return false;
                w.expert = share ? place / 8 / share : place / of_expert;
                i = share ? place % 8 * share + place / 8 % share : place % of_expert;
                if (i < of_expert) break;
            }
            place += gridDim.x;
            uint32_t row, column, lo, hi;
            grouped(i, p.row_tiles, p.col_tiles, row, column);
            w.row = row * 256;
            w.rows = p.m - w.row;
            w.column = column * 256;
            uniform_rows(p, w.expert, lo, hi);
            w.first = lo;
            w.length = hi - lo;
            w.steps = (w.length + Rows::kRows - 1) / Rows::kRows;
        } else {
            uint32_t i;
            for (;; place += gridDim.x) {
                if (place / 8 >= (total + 7) / 8) return false;
                if (tile_of(place, total, i)) break;
            }
            place += gridDim.x;
            const uint32_t l = fresh_thread() % 64;
            uint32_t upto = 0;   // experts whose first item is i or before
            for (uint32_t e = 0; e < p.experts; e += 64)
                upto += __popcll(__builtin_amdgcn_ballot_w64(e + l < p.experts && first[e + l] <= i));
            w.expert = __builtin_amdgcn_readfirstlane(upto - 1);
            i -= __builtin_amdgcn_readfirstlane(first[w.expert]);
            uint32_t lo, hi, row, column;
            uniform_rows(p, w.expert, lo, hi);
            const uint32_t whole = whole_tiles(hi - lo);
            if (i < whole * p.col_tiles) {
                grouped(i, whole, p.col_tiles, row, column);
            } else {
                const uint32_t s = span((hi - lo) % 256);
                row = whole;
                column = (i - whole * p.col_tiles) * s;
                columns_left = p.col_tiles - column < s ? p.col_tiles - column - 1 : s - 1;
            }
            w.row = lo + row * 256;
            w.rows = hi - w.row;
            w.column = column * 256;
            w.length = p.k * P::kSize;
            w.steps = (w.length + 127) / 128;
        }
        return true;
    };

    Rows rows;
    Columns columns;
    const lds_bytes r0 = (lds_bytes)rows0, r1 = (lds_bytes)rows1;
    const lds_bytes c0 = (lds_bytes)columns0, c1 = (lds_bytes)columns1;
    const uint32_t column_length = ACROSS ? p.k : 0;
    // operands of a tile, and its first two steps on their way
    auto begin = [&](const WideTile &w) {
        if (w.steps == 0) return;
        const uint32_t tid = fresh_thread();
        const uint32_t along = ACROSS && !GRAD ? column_length : w.length;
        if constexpr (GRAD) {
            const uint32_t lo = w.first;
            rows.start(p.row + lo * p.row_stride + (uint64_t)w.row * P::kSize, p.row_stride, w.rows,
                       w.length, tid);
            columns.start(p.col + lo * p.col_stride + (uint64_t)w.column * P::kSize, p.col_stride,
                          p.n - w.column, w.length, tid);
        } else {
            rows.start(p.row + w.row * p.row_stride, p.row_stride, w.rows, w.length, tid);
            columns.start(p.col + w.expert * p.col_expert +
                              w.column * (ACROSS ? (uint64_t)P::kSize : p.col_stride),
                          p.col_stride, p.n - w.column, along, tid);
        }
        rows.template load<false>(0, w.length, r0);
        columns.template load<false>(0, along, c0);
        if (w.steps > 1) {
            rows.template load<false>(1, w.length, r1);
            columns.template load<false>(1, along, c1);
        }
    };

    WideTile w, ahead;
    bool more = next(w);
    if (more) begin(w);
    uint32_t behind = 0;   // stores of the last tile's results
    while (more) {
        ahead = w;
        more = next(ahead);
        // the tile by RB blocks of 32 rows a wave
        auto run = [&](auto blocks) {
            constexpr int RB = decltype(blocks)::value;
            f32x16 acc[RB][4];
            const uint32_t l = fresh_thread() % 64, h = l / 32;
            constexpr int kReads = RB * Rows::kReads + 4 * Columns::kReads, kMma = RB * 4 * (P::kSize == 4 ? 4 : 1);
            const uint32_t whole = GRAD ? w.length / Rows::kRows : w.length / 128;
            const uint32_t along = ACROSS && !GRAD ? column_length : w.length;
            u32x4 rf[2][RB], cf[2][4];
            uint32_t re[2][RB], ce[2][4];   // mx4: exponents of a step
            // where they lie: this lane's rows and columns
            uint32_t re_at[RB], ce_at[4];
            const char *re_base = nullptr, *ce_base = nullptr;
            if constexpr (kMx4) {
                re_base = p.row_scale + w.row * p.row_scale_stride + 4 * h;
                ce_base = p.col_scale + w.expert * p.col_scale_expert + w.column * p.col_scale_stride + 4 * h;
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const uint32_t row = (wr * RB + r) * 32 + l % 32;
                    re_at[r] = (row < w.rows ? row : w.rows - 1) * (uint32_t)p.row_scale_stride;
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint32_t col = (wc * 4 + c) * 32 + l % 32;
                    ce_at[c] = (col < p.n - w.column ? col : p.n - w.column - 1) * (uint32_t)p.col_scale_stride;
                }
            }
            auto exponents = [&](uint32_t t, int to) {
                if constexpr (kMx4) {
                    const uint32_t count = w.length / 16;   // of a row
                    auto one = [&](const char *from, uint32_t at) {
                        if (t * 8 + 8 <= count)
                            return *(const __attribute__((address_space(1))) u32_any *)((global_bytes)from + t * 8 + at);
                        uint32_t v = 0;
#pragma unroll
                        for (uint32_t j = 0; j < 4; ++j)
                            if (t * 8 + 4 * h + j < count) v |= (uint32_t)(uint8_t)from[at + t * 8 + j] << (8 * j);
                        return v;
                    };
#pragma unroll
                    for (int r = 0; r < RB; ++r) re[to][r] = one(re_base, re_at[r]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) ce[to][c] = one(ce_base, ce_at[c]);
                }
            };
            auto read = [&](auto sub, lds_bytes rs, lds_bytes cs, int to) {
                constexpr int S = decltype(sub)::value;
                // in the order in which they are used
                cf[to][0] = Columns::fragment(cs, wc * 4, S, l);
                rf[to][0] = Rows::fragment(rs, wr * RB, S, l);
#pragma unroll
                for (int c = 1; c < 4; ++c) cf[to][c] = Columns::fragment(cs, wc * 4 + c, S, l);
#pragma unroll
                for (int r = 1; r < RB; ++r) rf[to][r] = Rows::fragment(rs, wr * RB + r, S, l);
            };
            auto mma = [&](auto sub, int f, int e) {
                constexpr int S = decltype(sub)::value;
#pragma unroll
                for (int r = 0; r < RB; ++r)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if constexpr (kMx4)
                            acc[r][c] = multiply_mx4<S>(cf[f][c], rf[f][r], ce[e][c], re[e][r], acc[r][c]);
                        else
                            acc[r][c] = multiply<P>(cf[f][c], rf[f][r], acc[r][c]);
                    }
            };
            using I0 = std::integral_constant<int, 0>;
            using I1 = std::integral_constant<int, 1>;
            using I2 = std::integral_constant<int, 2>;
            using I3 = std::integral_constant<int, 3>;
            // step t in (rt, ct), its first fragments read; E: which exponents are its own
            // FULL: two whole steps follow; kind 2: so for the first step
            auto body = [&](auto kind, auto parity, uint32_t t, lds_bytes rt, lds_bytes ct,
                            lds_bytes rn, lds_bytes cn) {
                constexpr bool FULL = decltype(kind)::value != 0, FIRST = decltype(kind)::value == 2;
                constexpr int E = decltype(parity)::value;
                constexpr int kScales = kMx4 ? RB + 4 : 0;
                if (FULL || t + 1 < w.steps) exponents(t + 1, 1 - E);
                read(I1{}, rt, ct, 1);
                mma(I0{}, 0, E);
                if constexpr (FULL) interleave<kReads, kMma, kScales, 0>();
                __builtin_amdgcn_sched_barrier(0);
                // the rows of the next step, fetched a step ago, to LDS, and those of the
                // one after it on their way; the columns follow when their buffer is free,
                // so that loads never queue up
                if (FULL ? !FIRST : t && t + 1 < w.steps) rows.put(rn);
                read(I2{}, rt, ct, 0);
                mma(I1{}, 1, E);
                if constexpr (FULL) interleave<kReads, kMma, 0, FIRST ? 0 : 8>();
                __builtin_amdgcn_sched_barrier(0);
                if (FULL || t + 2 < w.steps) rows.template fetch<FULL>(t + 2, w.length);
                read(I3{}, rt, ct, 1);
                mma(I2{}, 0, E);
                if constexpr (FULL) interleave<kReads, kMma, 8, 0>();
                __builtin_amdgcn_sched_barrier(0);
                // this wave has read all of the step, and its part of the next is there:
                // all loads but the last fetch have ended (step 1 is there from the start)
                if constexpr (FULL && !FIRST) __asm__ volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
                else if constexpr (FIRST) __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                else if (t) __asm__ volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                else __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (FULL) {
                    columns.template load<true>(t + 2, along, ct);
                    read(I0{}, rn, cn, 0);
                    mma(I3{}, 1, E);
                    interleave<kReads, kMma, 8, 0>();
                    __builtin_amdgcn_sched_barrier(0);
                } else {
                    if (t + 2 < w.steps) columns.template load<false>(t + 2, along, ct);
                    if (t + 1 < w.steps) read(I0{}, rn, cn, 0);
                    mma(I3{}, 1, E);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[r][c] = f32x16{};
            if (w.steps) {
                exponents(0, 0);
                read(I0{}, r0, c0, 0);
            }
            uint32_t t = 0;
            if (whole > 3) {
                body(I2{}, I0{}, 0, r0, c0, r1, c1);
                body(I1{}, I1{}, 1, r1, c1, r0, c0);
                for (t = 2; t + 3 < whole; t += 2) {
                    body(I1{}, I0{}, t, r0, c0, r1, c1);
                    body(I1{}, I1{}, t + 1, r1, c1, r0, c0);
                }
            }
            for (; t < w.steps; t += 2) {
                body(I0{}, I0{}, t, r0, c0, r1, c1);
                if (t + 1 < w.steps) body(I0{}, I1{}, t + 1, r1, c1, r0, c0);
            }

            const WideTile done = w;
            w = ahead;
            if (more) begin(w);

            char *out = p.out + (GRAD ? done.expert * p.out_expert : 0) + done.row * p.out_stride;
            constexpr int kEs = O::kSize;
            // whole pieces of 16 bytes: a descriptor drops what lies outside
            const bool pieces = !ADD && p.n % (16 / kEs) == 0 && p.out_stride < kWideStride;
            if (pieces) {
                // Through LDS, 32 rows of 128 bytes at a time, so that stores are of whole
                // lines (32 bytes of a row each, straight from the registers: 6 % slower).
                // A wave's accesses to LDS happen in order, which is all that its own part
                // of it needs.
                const rsrc_t to = make_rsrc(out, kOutside);
                const lds_bytes mine = (lds_bytes)stage + wave * kStage;
                constexpr int kWidth = 128 / kEs;
                behind = RB * 4 * kEs;
#pragma unroll
                for (int r = 0; r < RB; ++r)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const lds_bytes put = mine + l % 32 * 144 + (kEs == 4 ? h * 16 : c % 2 * 64 + h * 8);
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            float v[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) v[j] = acc[r][c][4 * q + j];
                            if constexpr (kEs == 4)
                                *(__attribute__((address_space(3))) u32x4 *)(put + q * 32) =
                                    u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]),
                                          __float_as_uint(v[2]), __float_as_uint(v[3])};
                            else
                                *(__attribute__((address_space(3))) u32x2 *)(put + q * 16) =
                                    u32x2{pair_of(v[0], v[1], dtype_of<O>()), pair_of(v[2], v[3], dtype_of<O>())};
                        }
                        if (kEs == 2 && c % 2 == 0) continue;
                        __builtin_amdgcn_wave_barrier();
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint32_t row = j * 8 + l / 8, in_tile = (wr * RB + r) * 32 + row;
                            const uint32_t col = done.column + (wc * 4 + (kEs == 4 ? c : c - 1)) * 32 +
                                                 l % 8 * (kWidth / 8);
                            const u32x4 v = *(const __attribute__((address_space(3))) u32x4 *)(
                                mine + row * 144 + l % 8 * 16);
                            const bool in = in_tile < done.rows && col < p.n;
                            bstore<kStoreKeep>(v, to, in ? in_tile * (uint32_t)p.out_stride + col * kEs : kOutside);
                        }
                        __builtin_amdgcn_wave_barrier();
                    }
            } else {
                behind = 0;
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const uint32_t row = (wr * RB + r) * 32 + l % 32;
                    char *to = out + row * p.out_stride;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint32_t col = done.column + (wc * 4 + c) * 32 + 8 * q + 4 * h;
                            if (row >= done.rows || col >= p.n) continue;
                            const uint32_t n = p.n - col < 4 ? p.n - col : 4;
                            float v[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) v[j] = acc[r][c][4 * q + j];
                            if constexpr (ADD)
#pragma unroll
                                for (uint32_t j = 0; j < 4; ++j)
                                    if (j < n) v[j] += up1<O>(to, col + j);
                            store_four(to, col, n, v, dtype_of<O>());
                        }
                }
            }
        };
        // The loads of the first two steps are there when all but the stores behind them
        // are: memory operations end in order.
        if (behind == 64) __asm__ volatile("s_waitcnt vmcnt(63)" ::: "memory");
        else if (behind == 32) __asm__ volatile("s_waitcnt vmcnt(32)" ::: "memory");
        else if (behind == 16) __asm__ volatile("s_waitcnt vmcnt(16)" ::: "memory");
        else if (behind == 8) __asm__ volatile("s_waitcnt vmcnt(8)" ::: "memory");
        else __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        // at most a half or a quarter of the rows: the waves share them differently
        if (w.rows > 128) run(std::integral_constant<int, 4>{});
        else if (w.rows > 64) run(std::integral_constant<int, 2>{});
        else run(std::integral_constant<int, 1>{});
    }
}

template <class P, class O, bool GRAD, bool ACROSS, bool ADD>
hipError_t go_wide(ProductParams p, hipStream_t s)
{
    p.col_tiles = (p.n + 255) / 256;
    p.row_tiles = (p.m + 255) / 256;
    const uint64_t tiles = (GRAD ? (uint64_t)p.experts * p.row_tiles
                                 : p.rows / 256 + (p.rows < p.experts ? p.rows : p.experts)) * p.col_tiles;
    // a workgroup on every CU, which takes what there is in turns
    const uint64_t cus = device_cus();
    // even out what workgroups do where each has enough items (12 a CU: 678 us without, 653
    // with; 6 a CU: 755 and 892, an item more or less being a fifth of the time)
    p.spans = tiles >= 8 * cus;
    return launch_kernel(product_wide_kernel<P, O, GRAD, ACROSS, ADD>,
                         dim3(grid_of(tiles < cus ? (tiles + 7) / 8 * 8 : cus, kProductThreads)),
                         dim3(kProductThreads), 0, s, p);
}

template <class P, class O>
hipError_t launch_wide(const ProductParams &p, bool grad, bool across, hipStream_t s)
{
    if constexpr (P::kSize == 1) {
        return go_wide<P, O, false, false, false>(p, s);
    } else {
        if (grad)
            return p.add ? go_wide<P, O, true, true, true>(p, s) : go_wide<P, O, true, true, false>(p, s);
        return across ? go_wide<P, O, false, true, false>(p, s) : go_wide<P, O, false, false, false>(p, s);
    }
}

}  // namespace xred
