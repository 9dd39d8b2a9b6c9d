// xred_product_wide.hpp -- the experts' products in tiles of 256 x 256, for calls with
// enough rows to fill the chip with them.
//
// Bound by the matrix cores (32768 rows of 64 experts, 4096 x 2048 bf16: 0.55 TFLOP, 390 us at
// a large library product's rate, 621 to 645 here; one expert 1217 TFLOP/s; 128 x 128 tiles 1340 us).
//
// A workgroup of four waves has a CU to itself: each wave keeps 128 x 128 sums in its
// 256 accumulation registers, so that a fragment of either operand is used four times
// and LDS is read at half of its rate while the matrix cores run.  Two steps of k (128
// KB) are in LDS, one being multiplied, the next on its way: its columns by loads straight
// to LDS, into a buffer that is free once the step's last fragments are read, three quarters
// through it, its rows through registers, so that loads spread over the step (all straight
// to LDS: they queue up behind one another).  Fragments are read one sub-step ahead, one
// between every two matrix instructions.
//
// Buffer descriptors bound every load: what lies past the operand's rows, columns or k
// comes as zero, so ragged tiles run the same code.  A tile of at most 128 or 64 rows
// has a main loop of its own that does a half or a quarter of the products.
//
// mx4: exponents of two steps at a time lie in LDS beside the operands, each lane's own
// dword of four (32768 rows, 4096 x 4096: 430 to 470 us, 2.3 to 2.6 PFLOP/s; 128 x 128 tiles 1100).
//
// e4m3: a step is the 128 elements that share their scales.  Its sums are scaled by vector
// instructions, 16 for two matrix instructions, and join sums of binary32: a tile of 256 x
// 128 leaves registers for them, and three steps in LDS since each is half the work for as
// long a way from memory (29500 rows, 4096 x 4096: 853 us, 1.16 PFLOP/s; two steps and 256
// x 128 1070, 128 x 128 tiles 1196).
//
// Workgroups stay for several tiles.  The first two steps of the next tile are loaded
// before the results of the last one go out, through LDS beside the operands', in whole
// pieces of 128 bytes of rows (mx4: 64).
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

// N rows (along) or columns (across) of an operand, a tile's.
template <class P, bool ACROSS, int N>
struct WideOperand : Pieces<P, ACROSS, N> {
    using Base = Pieces<P, ACROSS, N>;
    static constexpr int kPieces = Base::kPieces, kRows = Base::kRows;

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
                       : (uint64_t)(items < N ? items - 1 : N - 1) * stride + length;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint32_t q = Base::slot(i, tid), row = Base::row_of(q), piece = Base::piece_of(q);
            const bool there = ACROSS ? piece * 16 < items * P::kSize : row < items;
            at[i] = there ? row * (uint32_t)stride + piece * 16 : kOutside;
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
        return Base::piece_of(Base::slot(i, threadIdx.x)) * 16 < length - t * 128 ? at[i] : kOutside;
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

    // Step t straight into LDS, or zeros without reading anything.
    __device__ __forceinline__ void load_if(bool there, uint32_t t, uint32_t length, lds_bytes to) const
    {
        const uint64_t left = bytes - t * step;
        const rsrc_t r = make_rsrc(base + t * step, there ? left < kOutside ? (uint32_t)left : kOutside : 0);
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                r, (__attribute__((address_space(3))) void *)(to + (wave * kPieces + i) * 1024), 16,
                (int)offset<false>(i, t, length), 0, 0, 0);
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
                to + Base::slot(i, threadIdx.x) * 16) = held[i];
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

// Columns of a tile.  e4m3's sums are scaled by vector instructions, which cannot reach
// the accumulation registers: half as many fit beside what else a wave holds.  (Its file
// is compiled so that matrix instructions write to the others too.)
template <class P>
constexpr int wide_columns() { return __is_same(P, PE4M3) ? 128 : 256; }

// O: the output's type.  ADD: onto what it holds (gradient).
// GRID: operands on the 16-byte grid, in whole pieces; others go through registers, which
// leaves none for a gradient's two (2480 us where 128 x 128 tiles take 2210).
template <class P, class O, bool GRAD, bool ACROSS, bool ADD, bool GRID>
__device__ __forceinline__ void product_wide(const ProductParams &p)
{
    constexpr int BN = wide_columns<P>();
    using Rows = std::conditional_t<GRID, WideOperand<P, GRAD, 256>, LooseOperand<P, GRAD, 256, uint32_t>>;
    using Columns = std::conditional_t<GRID, WideOperand<P, ACROSS, BN>, LooseOperand<P, ACROSS, BN, uint32_t>>;
    constexpr bool kMx4 = __is_same(P, PMx4), kE4M3 = __is_same(P, PE4M3), kScaled = kMx4 || kE4M3;
    constexpr int kThreads = kProductThreads, kWaves = kThreads / 64;
    constexpr int CB = BN / 64, kAcross = 2;   // a wave's blocks of columns, waves side by side
    __shared__ __attribute__((aligned(1024))) char rows0[32768], rows1[32768];
    __shared__ __attribute__((aligned(1024))) char columns0[BN * 128], columns1[BN * 128];
    // results of a wave on their way out: 32 rows of kChunk bytes, kPitch apart
    constexpr int kChunk = kMx4 ? 64 : 128, kPitch = kChunk + 16, kStage = 32 * kPitch;
    __shared__ __attribute__((aligned(1024))) char rows2[kE4M3 ? 32768 : kWaves * kStage];
    __shared__ __attribute__((aligned(1024))) char columns2[kE4M3 ? BN * 128 : 16];
    // e4m3: its third step's buffer, which is free when results leave
    char *const stage = rows2;
    constexpr int kHalf = kMx4 ? 8192 : 4096;
    // 16 bytes for each row, then for each column, twice: mx4's exponents of two steps;
    // e4m3's row scales of four
    __shared__ __attribute__((aligned(16))) char scales[kScaled ? 2 * kHalf : 16];   // as planes of dwords
    __shared__ uint32_t first[GRAD ? 1 : XRED_MAX_EXPERTS];   // tile of each expert
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t wr = wave / kAcross, wc = wave % kAcross;
    // Work comes in items: a tile, or (p.spans) as many columns' tiles of an expert's last
    // rows as take about as long, two or three if those rows are at most 128 or 64.
    auto span = [&](uint32_t rest) { return p.spans ? rest > 64 ? 2u : 3u : 1u; };
    auto whole_tiles = [](uint32_t n) { return n / 256 + (n % 256 > 128); };
    auto items_of = [&](uint32_t n) {   // of an expert with n rows
        const uint32_t rest = n % 256, s = span(rest);
        return whole_tiles(n) * p.col_tiles + (rest == 0 || rest > 128 ? 0 : (p.col_tiles + s - 1) / s);
    };
    uint32_t total;   // items
    // gradient: an expert's tiles are dealt to all XCDs where there are enough of them,
    // since experts' rows, and with them the tiles' lengths, differ
    const uint32_t of_expert = p.row_tiles * p.col_tiles, share = of_expert < 64 ? 0 : (of_expert + 7) / 8;
    if constexpr (GRAD) {
        total = share ? p.experts * share * 8 : p.experts * of_expert;
    } else {
        RowTiles<kThreads> all;
        all.start(p, (uint32_t *)stage, items_of);
#pragma unroll
        for (int j = 0; j < RowTiles<kThreads>::kEach; ++j)
            first[threadIdx.x * RowTiles<kThreads>::kEach + j] = all.first[j];
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
            w.column += BN;
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
            w.column = column * BN;
            uniform_rows(p, w.expert, lo, hi);
            w.first = lo;
            w.length = hi - lo;
            w.steps = (w.length + Rows::kRows - 1) / Rows::kRows;
        } else {
            const uint32_t l = fresh_thread() % 64;
            uint32_t i, lo, hi, row, column;
            for (;; place += gridDim.x) {
                if (place / 8 >= (total + 7) / 8) return false;
                if (!tile_of(place, total, i)) continue;
                uint32_t upto = 0;   // experts whose first item is i or before
                for (uint32_t e = 0; e < p.experts; e += 64)
                    upto += __popcll(__builtin_amdgcn_ballot_w64(e + l < p.experts && first[e + l] <= i));
                if (upto == 0) continue;
                w.expert = __builtin_amdgcn_readfirstlane(upto - 1);
                i -= __builtin_amdgcn_readfirstlane(first[w.expert]);
                uniform_rows(p, w.expert, lo, hi);
                // else offsets do not ascend, and the sum has overflowed
                if (i < items_of(hi - lo)) break;
            }
            place += gridDim.x;
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
            w.column = column * BN;
            w.length = p.k * P::kSize;
            w.steps = (w.length + 127) / 128;
        }
        return true;
    };

    Rows rows;
    Columns columns;
    const lds_bytes r0 = (lds_bytes)rows0, r1 = (lds_bytes)rows1;
    const lds_bytes c0 = (lds_bytes)columns0, c1 = (lds_bytes)columns1;
    const lds_bytes r2 = (lds_bytes)rows2, c2 = (lds_bytes)columns2;
    (void)r2, (void)c2;
    const uint32_t column_length = ACROSS ? p.k : 0;
    // Scales of group g: mx4's exponents of steps 2 g and 2 g + 1, e4m3's row scales of
    // steps 4 g to 4 g + 3, 16 bytes for each row and column, a thread each.  They go through
    // registers to their half of `scales`; what lies past a row's end is masked when it is
    // read, or not read.
    u32x4 scale_held[2];
    auto fetch_scales = [&](const WideTile &w, uint32_t g) {
        if constexpr (kScaled) {
            const uint32_t tid = fresh_thread(), count = kMx4 ? w.length / 16 : w.steps * 4;
            auto load = [&](const char *from, uint64_t stride, uint32_t items) {
                items = items < 256 ? items : 256;
                const rsrc_t r = make_rsrc(from, (uint32_t)((items - 1) * stride + count));
                return bload<kLoadKeep>(
                    r, tid < items ? __umul24(tid, (uint32_t)stride) + g * 16 : kOutside);
            };
            scale_held[0] = load(p.row_scale + w.row * p.row_scale_stride, p.row_scale_stride, w.rows);
            if constexpr (kMx4)
                scale_held[1] = load(p.col_scale + w.expert * p.col_scale_expert +
                                         w.column * p.col_scale_stride, p.col_scale_stride, p.n - w.column);
        }
    };
    // A dword of each row and column makes a plane of 256, those of the blocks of 32 that a
    // lane works on side by side: a lane reads its own at once (several reads would be
    // merged into one whose place the compiler no longer knows, and which waits for all
    // loads to LDS).
    auto put_scales = [&](uint32_t g) {
        if constexpr (kScaled) {
            const uint32_t tid = fresh_thread();
            const lds_bytes to = (lds_bytes)scales + g % 2 * kHalf + tid % 32 * 32 + tid / 32 * 4;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                *(__attribute__((address_space(3))) uint32_t *)(to + i * 1024) = scale_held[0][i];
                if constexpr (kMx4)
                    *(__attribute__((address_space(3))) uint32_t *)(to + 4096 + i * 1024) = scale_held[1][i];
            }
        }
    };
    // Of `blocks` blocks from block b on, in plane i of group g; base: rows 0, columns 4096.
    auto scales_at = [&](auto blocks, uint32_t g, uint32_t base, uint32_t i, uint32_t b, uint32_t l,
                         uint32_t *to) {
        constexpr int N = decltype(blocks)::value;
        const lds_bytes from = (lds_bytes)scales + g % 2 * kHalf + base + i * 1024 + l % 32 * 32 + b * 4;
        if constexpr (N == 4) {
            const u32x4 v = *(const __attribute__((address_space(3))) u32x4 *)from;
            to[0] = v[0], to[1] = v[1], to[2] = v[2], to[3] = v[3];
        } else if constexpr (N == 2) {
            const u32x2 v = *(const __attribute__((address_space(3))) u32x2 *)from;
            to[0] = v[0], to[1] = v[1];
        } else {
            to[0] = *(const __attribute__((address_space(3))) uint32_t *)from;
        }
    };
    // operands of a tile, and its first two steps on their way (!GRID: the first)
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
        if constexpr (!GRID) {
            rows.template fetch<false>(0, w.length);
            columns.template fetch<false>(0, along);
        } else {
            rows.template load<false>(0, w.length, r0);
            columns.template load<false>(0, along, c0);
            if (w.steps > 1) {
                rows.template load<false>(1, w.length, r1);
                columns.template load<false>(1, along, c1);
            }
        }
        fetch_scales(w, 0);
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
            f32x16 acc[RB][CB];
            const uint32_t l = fresh_thread() % 64, h = l / 32;
            uint32_t whole = GRAD ? w.length / Rows::kRows : w.length / 128;
            if (!GRID && ACROSS) whole = whole ? whole - 1 : 0;   // a step follows
            const uint32_t along = ACROSS && !GRAD ? column_length : w.length;
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int c = 0; c < CB; ++c) acc[r][c] = f32x16{};
            if constexpr (kE4M3) {
            // e4m3: a step is 128 elements of k, which share their scales.  The sums of a
            // block of rows come from the matrix cores in `part` and join acc, scaled, while
            // the next block's are on their way.
            // Half the work a step for as long a way from memory: three steps are in LDS.
            u32x4 rf[4], cf[4][CB];
            f32x16 part[CB];
            float row_scale[RB], column_scale = 0.0f, last_by = 0.0f;
            part[CB - 1] = f32x16{};
            // one for the tile and step, by the scalar cache: a vector load would not end
            // before the steps that were asked for ahead of it
            using Scalars = const __attribute__((address_space(4))) float *;
            const Scalars column_scales =
                (Scalars)(uintptr_t)(p.col_scale + w.expert * p.col_scale_expert +
                                     w.column / 128 * p.col_scale_stride);
            auto scales_of = [&](uint32_t t) {
                uint32_t v[RB];
                scales_at(blocks, t / 4, 0, t % 4, wr * RB, l, v);
#pragma unroll
                for (int r = 0; r < RB; ++r) row_scale[r] = __uint_as_float(v[r]);
            };
            auto read_columns = [&](lds_bytes cs, int half) {
#pragma unroll
                for (int s = 2 * half; s < 2 * half + 2; ++s)
#pragma unroll
                    for (int c = 0; c < CB; ++c) cf[s][c] = Columns::fragment(cs, wc * CB + c, s, l);
            };
            auto read_row = [&](lds_bytes rs, int r, int half) {
#pragma unroll
                for (int s = 2 * half; s < 2 * half + 2; ++s) rf[s] = Rows::fragment(rs, wr * RB + r, s, l);
            };
            auto join = [&](int r, int c, float by) {
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[r][c][j] = __builtin_fmaf(part[c][j], by, acc[r][c][j]);
                // here and not later, when there would be more products waiting to join
                __asm__ volatile("" : "+v"(acc[r][c]));
            };
            // step t in (rt, ct), the next in (rn, cn); FULL: three whole ones follow
            auto body = [&](auto kind, uint32_t t, lds_bytes rt, lds_bytes ct, lds_bytes rn, lds_bytes cn) {
                constexpr bool FULL = decltype(kind)::value != 0;
                const bool go_on = FULL || t + 1 < w.steps;
                const float next_scale = column_scales[go_on ? t + 1 : t];
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const bool last = r + 1 == RB;
                    if (last) {
                        if (t % 4 == 2 && t + 2 < w.steps) put_scales(t / 4 + 1);
                        // the step's fragments have been read, and the next step is there:
                        // all loads but those of the one after it have ended
                        if constexpr (FULL) __asm__ volatile("s_waitcnt vmcnt(12) lgkmcnt(0)" ::: "memory");
                        else __asm__ volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                        __builtin_amdgcn_s_barrier();
                        if (t % 4 == 0 && t + 4 < w.steps) fetch_scales(w, t / 4 + 1);
                        __builtin_amdgcn_sched_barrier(0);
                        if (FULL || t + 3 < w.steps) {
                            rows.template load<FULL>(t + 3, w.length, rt);
                            columns.template load<FULL>(t + 3, w.length, ct);
                        }
                    }
                    static_assert(CB == 2, "the order below");
                    const float by = row_scale[r] * column_scale;
                    part[0] = multiply_e4m3(cf[0][0], cf[1][0], rf[0], rf[1], f32x16{});
                    join((r + RB - 1) % RB, 1, last_by);
                    part[1] = multiply_e4m3(cf[0][1], cf[1][1], rf[0], rf[1], f32x16{});
                    if (!last) read_row(rt, r + 1, 0);
                    else if (go_on) read_row(rn, 0, 0), read_columns(cn, 0);
                    part[0] = multiply_e4m3(cf[2][0], cf[3][0], rf[2], rf[3], part[0]);
                    part[1] = multiply_e4m3(cf[2][1], cf[3][1], rf[2], rf[3], part[1]);
                    if (!last) read_row(rt, r + 1, 1);
                    else if (go_on) read_row(rn, 0, 1), read_columns(cn, 1), scales_of(t + 1);
                    join(r, 0, by);
                    last_by = by;
                    if constexpr (FULL) {
                        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x20, 4, 0);
                        __builtin_amdgcn_sched_group_barrier(0x2, 17, 0);
                        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
                        __builtin_amdgcn_sched_group_barrier(0x20, 4, 0);
                        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x20, 4, 0);
                        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                        __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
                        __builtin_amdgcn_sched_group_barrier(0x2, 18, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                column_scale = next_scale;
            };
            using I0 = std::integral_constant<int, 0>;
            using I1 = std::integral_constant<int, 1>;
            if (w.steps) {
                if (w.steps > 2) {
                    rows.template load<false>(2, w.length, r2);
                    columns.template load<false>(2, w.length, c2);
                }
                column_scale = column_scales[0];
                read_columns(c0, 0);
                read_columns(c0, 1);
                read_row(r0, 0, 0);
                read_row(r0, 0, 1);
                scales_of(0);
            }
            uint32_t t = 0;
            for (; t + 5 < whole; t += 3) {
                body(I1{}, t, r0, c0, r1, c1);
                body(I1{}, t + 1, r1, c1, r2, c2);
                body(I1{}, t + 2, r2, c2, r0, c0);
            }
            for (; t < w.steps; t += 3) {
                body(I0{}, t, r0, c0, r1, c1);
                if (t + 1 < w.steps) body(I0{}, t + 1, r1, c1, r2, c2);
                if (t + 2 < w.steps) body(I0{}, t + 2, r2, c2, r0, c0);
            }
            join(RB - 1, 1, last_by);
            } else {
            constexpr int kReads = RB * Rows::kReads + 4 * Columns::kReads, kMma = RB * 4 * (P::kSize == 4 ? 4 : 1);
            u32x4 rf[2][RB], cf[2][4];
            uint32_t re[2][RB], ce[2][4];   // mx4: exponents of a step
            // of step t, from `scales`; LAST: the row may end in it
            auto exponents = [&](auto last, uint32_t t, int to) {
                if constexpr (kMx4) {
                    const bool there = !decltype(last)::value || t * 8 + 4 * h < w.length / 16;
                    scales_at(blocks, t / 2, 0, t % 2 * 2 + h, wr * RB, l, re[to]);
                    scales_at(std::integral_constant<int, 4>{}, t / 2, 4096, t % 2 * 2 + h, wc * 4, l, ce[to]);
#pragma unroll
                    for (int r = 0; r < RB; ++r) re[to][r] = there ? re[to][r] : 0;
#pragma unroll
                    for (int c = 0; c < 4; ++c) ce[to][c] = there ? ce[to][c] : 0;
                }
            };
            auto read = [&](auto sub, lds_bytes rs, lds_bytes cs, int to) {
                constexpr int S = decltype(sub)::value;
                // in the order in which they are used
                cf[to][0] = Columns::fragment(cs, wc * CB, S, l);
                rf[to][0] = Rows::fragment(rs, wr * RB, S, l);
#pragma unroll
                for (int c = 1; c < 4; ++c) cf[to][c] = Columns::fragment(cs, wc * CB + c, S, l);
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
                constexpr bool FULL = decltype(kind)::value != 0, FIRST = GRID && decltype(kind)::value == 2;
                constexpr int E = decltype(parity)::value;
                if constexpr (kMx4 && E == 0)
                    if (FULL || t + 2 < w.steps) fetch_scales(w, t / 2 + 1);
                if constexpr (kMx4 && E == 1)
                    if (FULL || t + 1 < w.steps) put_scales(t / 2 + 1);
                read(I1{}, rt, ct, 1);
                mma(I0{}, 0, E);
                if constexpr (FULL) interleave<kReads, kMma, kMx4 && E == 0 ? 2 : 0, kMx4 && E == 1 ? 8 : 0>();
                __builtin_amdgcn_sched_barrier(0);
                // the rows of the next step, fetched a step ago, to LDS, and those of the
                // one after it on their way; the columns follow when their buffer is free,
                // so that loads never queue up
                if constexpr (GRID) {
                    if (FULL ? !FIRST : t && t + 1 < w.steps) rows.put(rn);
                } else if (FULL || t + 1 < w.steps) {
                    rows.template put<FULL>(t + 1, w.length, rn);
                    columns.template put<FULL>(t + 1, along, cn);
                }
                read(I2{}, rt, ct, 0);
                mma(I1{}, 1, E);
                if constexpr (FULL) interleave<kReads, kMma, 0, FIRST ? 0 : GRID ? 8 : 16>();
                __builtin_amdgcn_sched_barrier(0);
                if (FULL || t + 2 < w.steps) rows.template fetch<FULL>(t + 2, w.length);
                read(I3{}, rt, ct, 1);
                mma(I2{}, 0, E);
                if constexpr (FULL) interleave<kReads, kMma, 8, 0>();
                __builtin_amdgcn_sched_barrier(0);
                // this wave has read all of the step, and its part of the next is there:
                // all loads but the last fetch have ended (step 1 is there from the start)
                if constexpr (!GRID) __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                else if constexpr (FULL && !FIRST) __asm__ volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
                else if constexpr (FIRST) __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                else if (t) __asm__ volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                else __asm__ volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (FULL) {
                    if constexpr (GRID) columns.template load<true>(t + 2, along, ct);
                    else columns.template fetch<true>(t + 2, along);
                    read(I0{}, rn, cn, 0);
                    exponents(std::false_type{}, t + 1, 1 - E);
                    mma(I3{}, 1, E);
                    interleave<kReads + (kMx4 ? 2 : 0), kMma, 8, 0>();
                    __builtin_amdgcn_sched_barrier(0);
                } else {
                    if (t + 2 < w.steps) {
                        if constexpr (GRID) columns.template load<false>(t + 2, along, ct);
                        else columns.template fetch<false>(t + 2, along);
                    }
                    if (t + 1 < w.steps) {
                        read(I0{}, rn, cn, 0);
                        exponents(std::true_type{}, t + 1, 1 - E);
                    }
                    mma(I3{}, 1, E);
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            if (w.steps) {
                exponents(std::true_type{}, 0, 0);
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

            }

            const WideTile done = w;
            w = ahead;
            if (more) begin(w);

            char *out = p.out + (GRAD ? done.expert * p.out_expert : 0) + done.row * p.out_stride;
            constexpr int kEs = O::kSize;
            // whole pieces of 16 bytes: a descriptor drops what lies outside
            const bool pieces = !ADD && p.n % (16 / kEs) == 0 && p.out_stride < kWideStride;
            if (pieces) {
                // Through LDS, 32 rows of 64 or 128 bytes at a time, so that stores are of whole
                // lines (32 bytes of a row each, straight from the registers: 6 % slower).
                // A wave's accesses to LDS happen in order, which is all that its own part
                // of it needs.
                const rsrc_t to = make_rsrc(out, kOutside);
                const lds_bytes mine = (lds_bytes)stage + wave * kStage;
                constexpr int kWidth = kChunk / kEs, kLanes = kChunk / 16;   // of a row
                behind = RB * CB * kEs;
#pragma unroll
                for (int r = 0; r < RB; ++r)
#pragma unroll
                    for (int i = 0; i < 4 * CB; ++i) {   // 8 columns each
                        const int c = i / 4, q = i % 4, part = i % (kWidth / 8);
                        float v[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] = acc[r][c][4 * q + j];
                        const lds_bytes put = mine + l % 32 * kPitch + (part * 8 + h * 4) * kEs;
                        if constexpr (kEs == 4)
                            *(__attribute__((address_space(3))) u32x4 *)put =
                                u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]),
                                      __float_as_uint(v[2]), __float_as_uint(v[3])};
                        else
                            *(__attribute__((address_space(3))) u32x2 *)put =
                                u32x2{pair_of(v[0], v[1], dtype_of<O>()), pair_of(v[2], v[3], dtype_of<O>())};
                        if (part != kWidth / 8 - 1) continue;
                        __builtin_amdgcn_wave_barrier();
#pragma unroll
                        for (int j = 0; j < kLanes / 2; ++j) {
                            const uint32_t row = j * (64 / kLanes) + l / kLanes;
                            const uint32_t in_tile = (wr * RB + r) * 32 + row;
                            const uint32_t col = done.column + wc * (32 * CB) + (i + 1) * 8 - kWidth +
                                                 l % kLanes * (16 / kEs);
                            const u32x4 x = *(const __attribute__((address_space(3))) u32x4 *)(
                                mine + row * kPitch + l % kLanes * 16);
                            const bool in = in_tile < done.rows && col < p.n;
                            bstore<kStoreKeep>(x, to, in ? in_tile * (uint32_t)p.out_stride + col * kEs : kOutside);
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
                    for (int c = 0; c < CB; ++c)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint32_t col = done.column + (wc * CB + c) * 32 + 8 * q + 4 * h;
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
        else if (behind == 4) __asm__ volatile("s_waitcnt vmcnt(4)" ::: "memory");
        else __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (w.steps) {
            put_scales(0);
            if constexpr (!GRID) {
                const uint32_t along = ACROSS && !GRAD ? column_length : w.length;
                rows.template put<false>(0, w.length, r0);
                columns.template put<false>(0, along, c0);
                if (w.steps > 1) {
                    rows.template fetch<false>(1, w.length);
                    columns.template fetch<false>(1, along);
                }
            }
        }
        __syncthreads();
        // at most a half or a quarter of the rows: the waves share them differently
        if (w.rows > 128) run(std::integral_constant<int, 4>{});
        else if (w.rows > 64) run(std::integral_constant<int, 2>{});
        else run(std::integral_constant<int, 1>{});
    }
}

template <class P, class O, bool GRAD, bool ACROSS, bool ADD, bool GRID>
__global__ __launch_bounds__(kProductThreads, 1) void product_wide_kernel(ProductParams p)
{
    product_wide<P, O, GRAD, ACROSS, ADD, GRID>(p);
}

template <class P, class O, bool GRAD, bool ACROSS, bool ADD, bool GRID>
hipError_t go_wide(ProductParams p, hipStream_t s)
{
    constexpr uint32_t BN = wide_columns<P>();
    p.col_tiles = (p.n + BN - 1) / BN;
    p.row_tiles = (p.m + 255) / 256;
    const uint64_t tiles = (GRAD ? (uint64_t)p.experts * p.row_tiles
                                 : p.rows / 256 + (p.rows < p.experts ? p.rows : p.experts)) * p.col_tiles;
    p.most = (uint32_t)tiles;
    // a workgroup on every CU, which takes what there is in turns
    const uint64_t cus = device_cus();
    // even out what workgroups do where each has enough items (12 a CU: 678 us without, 653
    // with; 6 a CU: 755 and 892, an item more or less being a fifth of the time)
    p.spans = tiles >= 8 * cus;
    return launch_kernel(product_wide_kernel<P, O, GRAD, ACROSS, ADD, GRID>,
                         dim3(grid_of(tiles < cus ? (tiles + 7) / 8 * 8 : cus, kProductThreads)),
                         dim3(kProductThreads), 0, s, p);
}

template <class P, class O>
hipError_t launch_wide(const ProductParams &p, bool grad, bool across, hipStream_t s)
{
    if constexpr (P::kSize == 1) {
        return go_wide<P, O, false, false, false, true>(p, s);
    } else {
        if constexpr (P::kSize == 2)
            if (grad)
                return p.add ? go_wide<P, O, true, true, true, true>(p, s)
                             : go_wide<P, O, true, true, false, true>(p, s);
        return across ? go_wide<P, O, false, true, false, true>(p, s)
                      : go_wide<P, O, false, false, false, true>(p, s);
    }
}

}  // namespace xred
