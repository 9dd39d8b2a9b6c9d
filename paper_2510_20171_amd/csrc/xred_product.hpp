// xred_product.hpp -- the experts' matrix products over ragged rows on the matrix
// cores: device code of xred_group_product and xred_group_product_grad.
//
// Both are tiles of D[row][column] = sum over k of R[row][k] * C[column][k], where R
// and C are two operands whose rows lie along k, or across it (k counts their rows):
//     forward     R = x (along),      C = w (along; across when transposed)
//     gradient    R = dout (across),  C = x (across), k an expert's rows
// Operand bytes go through LDS in steps of 128 bytes of k for each row (64 elements
// of 2 bytes, 32 of fp32, 128 of e4m3, 256 of mx4), so that every type runs the same
// code around its matrix instruction.
//
// Layout of a step in LDS: along, each row's eight 16-byte pieces in order of
// piece ^ (row % 8), so that eight neighbouring rows' pieces of one place lie in
// different banks; across, rows of k as they lie in memory, 16-bit ones in pairs of
// pieces in order of pair ^ (row % 4), for the transposing reads.
//
// A fragment is 16 bytes of a lane: lane l holds row l % 32 of a block of 32 and, in
// sub-step s of four, piece 4 * (l / 32) + s of the step.  Any order of k serves, as
// long as both operands keep to it; this one gives a lane the dword of an mx4 row's
// eight exponents that its pieces need.
#pragma once

#include "xred_product_launch.hpp"
#include "xred_rows.hpp"

namespace xred {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char *lds_bytes;

// Operand types: bytes of an element (mx4: of two), elements of k in a step.
struct PBF16 {
    static constexpr int kSize = 2, kStep = 64;
};
struct PF16 {
    static constexpr int kSize = 2, kStep = 64;
};
struct PF32 {
    static constexpr int kSize = 4, kStep = 32;
};
struct PE4M3 {
    static constexpr int kSize = 1, kStep = 128;
};
struct PMx4 {
    static constexpr int kSize = 1, kStep = 128;   // counted in bytes
};

// The element type of an unscaled operand, as an output's.
template <class P> struct OwnType;
template <> struct OwnType<PBF16> { using T = TBF16; };
template <> struct OwnType<PF16> { using T = TF16; };
template <> struct OwnType<PF32> { using T = TF32; };

constexpr int kProductThreads = 256;

// acc += columns' fragment (32 columns) * rows' fragment (32 rows): lane l has row
// l % 32 and, in registers 4 q .. 4 q + 3, columns 8 q + 4 (l / 32) and the next three.
template <class P>
__device__ __forceinline__ f32x16 multiply(u32x4 c, u32x4 r, f32x16 acc)
{
    if constexpr (__is_same(P, PBF16)) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, c),
                                                       __builtin_bit_cast(bf16x8, r), acc, 0, 0, 0);
    } else if constexpr (__is_same(P, PF16)) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, c),
                                                      __builtin_bit_cast(f16x8, r), acc, 0, 0, 0);
    } else {
        static_assert(__is_same(P, PF32));
#pragma unroll
        for (int j = 0; j < 4; ++j)
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(c[j]), __uint_as_float(r[j]),
                                                       acc, 0, 0, 0);
        return acc;
    }
}

__device__ __forceinline__ i32x8 two(u32x4 a, u32x4 b)
{
    return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

// Two fragments of e4m3, 64 elements of k, times 1 (the exponent 127 in every byte).
__device__ __forceinline__ f32x16 multiply_e4m3(u32x4 c0, u32x4 c1, u32x4 r0, u32x4 r1, f32x16 acc)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(two(c0, c1), two(r0, r1), acc, 0, 0, 0,
                                                           0x7F7F7F7F, 0, 0x7F7F7F7F);
}

// A fragment of e2m1, 64 elements of k; byte S of cs and rs holds the exponents.
template <int S>
__device__ __forceinline__ f32x16 multiply_mx4(u32x4 c, u32x4 r, uint32_t cs, uint32_t rs, f32x16 acc)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(two(c, u32x4{}), two(r, u32x4{}), acc, 4,
                                                           4, S, (int)cs, S, (int)rs);
}

// What loads past the end of k read instead.
__device__ const u32x4 product_zeros = {0, 0, 0, 0};

// ---------------------------------------------------------------- operands --
// The operand of a tile's N rows (along) or columns (across), in pieces of 16 bytes,
// kPieces a thread and step.
template <class P, bool ACROSS, int N>
struct Pieces {
    static constexpr int kPieces = N * 128 / 16 / kProductThreads;
    static constexpr int kWide = N * P::kSize / 16;   // across: pieces of a row of k
    static constexpr int kRows = 128 / P::kSize;      // across: rows of k in a step
    static constexpr int kReads = ACROSS ? (P::kSize == 2 ? 2 : 4) : 1;   // of LDS for a fragment

    // Place i in LDS of thread tid, in pieces; what lies there: a row, and a piece of it.
    static __device__ __forceinline__ uint32_t slot(int i, uint32_t tid)
    {
        return (tid / 64 * kPieces + i) * 64 + tid % 64;
    }
    static __device__ __forceinline__ uint32_t row_of(uint32_t q) { return ACROSS ? q / kWide : q / 8; }
    static __device__ __forceinline__ uint32_t piece_of(uint32_t q)
    {
        if constexpr (!ACROSS) return q % 8 ^ q / 8 % 8;
        const uint32_t piece = q % kWide;
        return P::kSize == 2 ? piece ^ q / kWide % 4 * 2 : piece;
    }

    // Sub-step s of block b of 32.
    static __device__ __forceinline__ u32x4 fragment(lds_bytes from, int b, int s,
                                                     uint32_t l = threadIdx.x % 64)
    {
        const uint32_t h = l / 32;
        if constexpr (!ACROSS) {
            return *(const __attribute__((address_space(3))) u32x4 *)(
                from + b * 4096 + l % 32 * 128 + ((4 * h + s) ^ l % 8) * 16);
        } else if constexpr (P::kSize == 2) {
            // 16 lanes read 4 rows of 16 columns: lane i gets column i of them
            const uint32_t i = l % 16, row = 8 * (4 * h + s) + i / 4;
            const uint32_t piece = (b * 4 + l / 16 % 2 * 2 + i % 4 / 2) ^ (i / 4 * 2);
            const lds_bytes p = from + row * (N * 2) + piece * 16 + i % 2 * 8;
            using Read = __attribute__((address_space(3))) i16x4 *;
            const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Read)p));
            const u32x2 c = __builtin_bit_cast(
                u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Read)(p + 4 * N * 2)));
            return u32x4{a[0], a[1], c[0], c[1]};
        } else {
            static_assert(P::kSize == 4);
            const lds_bytes p = from + 4 * (4 * h + s) * (N * 4) + (b * 32 + l % 32) * 4;
            u32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] = *(const __attribute__((address_space(3))) uint32_t *)(p + j * (N * 4));
            return v;
        }
    }
};

// An operand whose pieces lie on the 16-byte grid, whole ones only: straight to LDS.
template <class P, bool ACROSS, int N>
struct GridOperand : Pieces<P, ACROSS, N> {
    using Base = Pieces<P, ACROSS, N>;
    static constexpr int kPieces = Base::kPieces, kRows = Base::kRows;
    const char *base;
    uint64_t step;            // bytes from one step to the next
    uint64_t at[kPieces];     // from base: this thread's pieces

    // items: rows (along) or columns (across) that exist, at least one; those
    // behind them are read as others, whose products nobody stores.
    __device__ __forceinline__ void start(const char *from, uint64_t stride, uint32_t items, uint32_t)
    {
        base = from;
        step = ACROSS ? stride * kRows : 128;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint32_t q = Base::slot(i, threadIdx.x), row = Base::row_of(q), at16 = Base::piece_of(q) * 16;
            if constexpr (ACROSS) at[i] = row * stride + (at16 < items * P::kSize ? at16 : 0);
            else at[i] = (row < items ? row : items - 1) * stride + at16;
        }
    }

    // Step t of k to `to`.  length: of k, in bytes (along) or rows (across).
    __device__ __forceinline__ void load(uint32_t t, uint32_t length, lds_bytes to)
    {
        const uint32_t left = length - t * (ACROSS ? kRows : 128);
        const bool whole = left >= (ACROSS ? kRows : 128);
        const char *from = base + t * step;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const char *src = from + at[i];
            const uint32_t q = Base::slot(i, threadIdx.x);
            if (!whole && (ACROSS ? Base::row_of(q) : Base::piece_of(q) * 16) >= left)
                src = (const char *)&product_zeros;
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void *)src,
                (__attribute__((address_space(3))) void *)(to + (threadIdx.x / 64 * kPieces + i) * 1024),
                16, 0, 0);
        }
    }
    __device__ __forceinline__ void store(uint32_t, uint32_t, lds_bytes) const {}
};

// Bytes [skip, skip + n) of v, zeros behind them.
__device__ __forceinline__ u32x4 bytes_of(u32x4 v, uint32_t skip, uint32_t n)
{
    uint64_t lo = v[0] | (uint64_t)v[1] << 32, hi = v[2] | (uint64_t)v[3] << 32;
    if (skip >= 8) lo = hi, hi = 0, skip -= 8;
    if (skip >= 8) lo = 0;
    else if (skip) lo = lo >> 8 * skip | hi << (64 - 8 * skip), hi >>= 8 * skip;
    if (n < 8) lo &= ((uint64_t)1 << 8 * n) - 1, hi = 0;
    else if (n < 16) hi &= ((uint64_t)1 << 8 * (n - 8)) - 1;
    return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// An operand at any element, of any length: by way of registers.  A piece is read whole,
// with what follows it in memory; only in the operand's last steps does that matter, where
// a piece past the end is read as its last 16 bytes, shifted into place, and what is past
// the end of k becomes zero.  Offset: of an offset within a step.
template <class P, bool ACROSS, int N, class Offset>
struct LooseOperand : Pieces<P, ACROSS, N> {
    using Base = Pieces<P, ACROSS, N>;
    static constexpr int kPieces = Base::kPieces, kRows = Base::kRows;
    const char *base;
    uint64_t step, bytes;   // from one step to the next; from base to the operand's end
    Offset at[kPieces];
    u32x4 held[kPieces];

    // length: of k, in bytes (along) or rows (across), at least one.
    __device__ __forceinline__ void start(const char *from, uint64_t stride, uint32_t items,
                                          uint32_t length, uint32_t tid = threadIdx.x)
    {
        base = from;
        step = ACROSS ? stride * kRows : 128;
        bytes = ACROSS ? (length - 1) * stride + (uint64_t)items * P::kSize
                       : (uint64_t)(items - 1) * stride + length;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint32_t q = Base::slot(i, tid), row = Base::row_of(q), at16 = Base::piece_of(q) * 16;
            if constexpr (ACROSS) at[i] = row * (Offset)stride + (at16 < items * P::kSize ? at16 : 0);
            else at[i] = (row < items ? row : items - 1) * (Offset)stride + at16;
        }
    }

    // Where piece i of step t begins; false: past the end of k.  left: bytes of it before that
    __device__ __forceinline__ bool place(int i, uint32_t t, uint32_t length, uint64_t &off, uint32_t &left) const
    {
        const uint32_t q = Base::slot(i, threadIdx.x);
        const uint32_t k = t * (ACROSS ? kRows : 128) + (ACROSS ? Base::row_of(q) : Base::piece_of(q) * 16);
        left = ACROSS ? 16 : length - k;
        off = t * step + at[i];
        return k < length;
    }

    // WHOLE: step t ends before the last row of k (across) or a row's end (along).
    template <bool WHOLE>
    __device__ __forceinline__ void fetch(uint32_t t, uint32_t length)
    {
        using Vec = const __attribute__((address_space(1))) u32x4_any;
        if constexpr (WHOLE) {
            const char *from = base + t * step;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) held[i] = *(Vec *)((global_bytes)from + at[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                uint64_t off;
                uint32_t left;
                if (!place(i, t, length, off, left)) {
                    held[i] = u32x4{0, 0, 0, 0};
                } else if (bytes >= 16) {
                    held[i] = *(Vec *)((global_bytes)base + (off < bytes - 16 ? off : bytes - 16));
                } else {   // an operand of a few elements, byte by byte
                    uint64_t lo = 0, hi = 0;
#pragma clang loop unroll(disable)
                    for (uint64_t j = off < bytes ? bytes - off : 0; j-- > 0;) {
                        hi = hi << 8 | lo >> 56;
                        lo = lo << 8 | (uint8_t)base[off + j];
                    }
                    held[i] = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
                }
            }
        }
    }
    template <bool WHOLE>
    __device__ __forceinline__ void put(uint32_t t, uint32_t length, lds_bytes to) const
    {
        put<WHOLE>(t, length, to, held);
    }
    // The same of pieces kept elsewhere.  An operand of at least 16 bytes, whatever the step:
    // no branch, so that the compiler can count what is on its way.
    __device__ __forceinline__ void fetch_any(uint32_t t, u32x4 (&v)[kPieces]) const
    {
        const uint64_t from = t * step, most = bytes - 16;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint64_t off = from + at[i];
            v[i] = *(const __attribute__((address_space(1))) u32x4_any *)((global_bytes)base + (off < most ? off : most));
        }
    }
    template <bool WHOLE>
    __device__ __forceinline__ void put(uint32_t t, uint32_t length, lds_bytes to, const u32x4 (&pieces)[kPieces]) const
    {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            u32x4 v = pieces[i];
            if constexpr (!WHOLE) {
                uint64_t off;
                uint32_t left;
                const bool there = place(i, t, length, off, left);
                const uint64_t skip = bytes >= 16 && off > bytes - 16 ? off - (bytes - 16) : 0;
                v = bytes_of(v, skip < 16 ? (uint32_t)skip : 16, !there ? 0 : left < 16 ? left : 16);
            }
            *(__attribute__((address_space(3))) u32x4 *)(to + Base::slot(i, threadIdx.x) * 16) = v;
        }
    }
    // Whether step t is whole, and rows of at least 16 bytes follow.
    static __device__ __forceinline__ bool is_whole(uint32_t t, uint32_t length)
    {
        return ACROSS ? (t + 2) * kRows <= length : (t + 1) * 128 <= length;
    }
    __device__ __forceinline__ void load(uint32_t t, uint32_t length, lds_bytes)
    {
        if (is_whole(t, length)) fetch<true>(t, length);
        else fetch<false>(t, length);
    }
    __device__ __forceinline__ void store(uint32_t t, uint32_t length, lds_bytes to) const
    {
        if (is_whole(t, length)) put<true>(t, length, to);
        else put<false>(t, length, to);
    }
};

// ------------------------------------------------------------------- tiles --
// Rows of expert e, whatever the offsets hold.
__device__ __forceinline__ void expert_rows(const ProductParams &p, uint32_t e, uint32_t &lo, uint32_t &hi)
{
    const int32_t a = p.offsets[e], b = p.offsets[e + 1];
    lo = a < 0 ? 0u : (uint32_t)a < p.rows ? (uint32_t)a : p.rows;
    hi = b < (int32_t)lo ? lo : (uint32_t)b < p.rows ? (uint32_t)b : p.rows;
}

// Tiles of BM rows over all experts, in their order; a thread keeps a few experts.
template <int THREADS>
struct RowTiles {
    static constexpr int kEach = XRED_MAX_EXPERTS / THREADS;
    uint32_t lo[kEach], hi[kEach], first[kEach], tiles[kEach];
    uint32_t total;

    // tiles_of(n): of an expert with n rows.  shared: THREADS / 64 words.  Ends with a
    // barrier.
    template <class F>
    __device__ __forceinline__ void start(const ProductParams &p, uint32_t *shared, F &&tiles_of)
    {
        uint32_t own = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const uint32_t e = threadIdx.x * kEach + j;
            lo[j] = hi[j] = 0;
            if (e < p.experts) expert_rows(p, e, lo[j], hi[j]);
            tiles[j] = tiles_of(hi[j] - lo[j]);
            first[j] = own;
            own += tiles[j];
        }
        uint32_t before, all;
        lanes_before<64>(own, before, all);
        if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = all;
        __syncthreads();
        total = 0;
#pragma unroll
        for (uint32_t w = 0; w < THREADS / 64; ++w) {
            before += w < threadIdx.x / 64 ? shared[w] : 0;
            total += shared[w];
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) first[j] += before;
        // offsets out of order: a workgroup's places must not wrap round on the way there
        total = total < p.most ? total : p.most;
    }

    // Tile t (below total): its expert and rows [lo, hi), into found[3] (LDS).  Offsets that do
    // not ascend can make the sum overflow, and then none is found.
    __device__ __forceinline__ void find(uint32_t t, uint32_t rows_of_tile, uint32_t *found) const
    {
        __syncthreads();   // the tile before has been read
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (t - first[j] < tiles[j]) {
                found[0] = threadIdx.x * kEach + j;
                found[1] = lo[j] + (t - first[j]) * rows_of_tile;
                found[2] = hi[j];
            }
        __syncthreads();
    }
};

// Place i of a launch to a tile: workgroups i, i + 8, ... run on one XCD, and get
// neighbouring tiles, whose operands its L2 then holds; false: none.
__device__ __forceinline__ bool tile_of(uint32_t i, uint32_t total, uint32_t &tile)
{
    const uint32_t share = (total + 7) / 8;
    tile = i % 8 * share + i / 8;
    return i / 8 < share && tile < total;
}

// Two values of bf16 or fp16 as a word.
__device__ __forceinline__ uint32_t pair_of(float a, float b, xred_dtype type)
{
    if (type == XRED_BFLOAT16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
    const uint32_t lo = __builtin_bit_cast(uint16_t, (_Float16)a);
    return lo | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)b) << 16;
}

// Four output values from column c on, n of them.
__device__ __forceinline__ void store_four(char *row, uint32_t c, uint32_t n, const float (&v)[4],
                                           xred_dtype type)
{
    if (type == XRED_FLOAT32) {
        if (n == 4) {
            *(__attribute__((address_space(1))) u32x4_any *)((global_out)row + c * 4ull) =
                u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                      __float_as_uint(v[3])};
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j)
                if (j < n) down1<TF32, OpSum>(row, c + j, v[j]);
        }
        return;
    }
    const u32x2 w = {pair_of(v[0], v[1], type), pair_of(v[2], v[3], type)};
    if (n == 4) {
        *(__attribute__((address_space(1))) u32x2_any *)((global_out)row + c * 2ull) = w;
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            if (j < n) ((uint16_t *)row)[c + j] = (uint16_t)(w[j / 2] >> (16 * (j % 2)));
    }
}

__device__ __forceinline__ float value_at(const char *row, uint32_t c, xred_dtype type)
{
    return type == XRED_FLOAT32 ? up1<TF32>(row, c)
         : type == XRED_BFLOAT16 ? up1<TBF16>(row, c) : up1<TF16>(row, c);
}

// ------------------------------------------------------------------ kernel --
// 4 waves, two by two, each RB x CB blocks of 32 x 32: tiles of 64 RB x 64 CB, one step of
// k multiplied while the next is on its way.  What the wider and the narrower tiles do not
// take: n or k below 64, rows 8 MB and more apart, fp32 but for thousands of tiles, gradients of
// few tiles or off the 16-byte grid, forward products with fewer tiles than the wider ones need.
// Bound by that way from memory (32768 rows, 4096 x 2048 bf16 would take 1340 us, 410
// TFLOP/s; the gradient of 515 x 1027 fp32, 8 experts, 1800 rows 40 us, 18 of them matrix
// instructions).
// Two of the larger tiles or four of the smaller have to fit a CU: while one waits for its
// loads, another multiplies (one: 4200 us where two take 2210; with HALVES, rare, two).
//
// HALVES: each half of the steps, sub-steps 0 and 1 and sub-steps 2 and 3, has sums of its own,
// which meet at the end, as in the streaming tiles (xred_product_narrow.hpp), in whose place
// these take rows 8 MB and more apart: the same bits at any distance.
template <class P, bool GRAD, bool ACROSS, bool DIRECT, int RB, int CB, bool HALVES>
__global__ __launch_bounds__(kProductThreads, RB == 2 || HALVES ? 2 : 4) void product_kernel(ProductParams p)
{
    constexpr int BM = 64 * RB, BN = 64 * CB;
    using Rows = std::conditional_t<DIRECT, GridOperand<P, GRAD, BM>, LooseOperand<P, GRAD, BM, uint64_t>>;
    using Columns = std::conditional_t<DIRECT, GridOperand<P, ACROSS, BN>, LooseOperand<P, ACROSS, BN, uint64_t>>;
    // two steps, each an array of its own: a read of one does not wait for loads into
    // the other
    __shared__ __attribute__((aligned(1024))) char rows0[BM * 128], rows1[BM * 128];
    __shared__ __attribute__((aligned(1024))) char columns0[BN * 128], columns1[BN * 128];
    __shared__ uint32_t shared[kProductThreads / 64], found[3];
    const uint32_t l = threadIdx.x % 64, h = l / 32;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t wr = wave / 2, wc = wave % 2;   // this wave's place
    RowTiles<kProductThreads> all;
    uint32_t total;
    // gradient: an expert's tiles are dealt to all XCDs where there are enough of them,
    // since experts' rows, and with them the tiles' lengths, differ
    const uint32_t of_expert = p.row_tiles * p.col_tiles, share = of_expert < 64 ? 0 : (of_expert + 7) / 8;
    if constexpr (GRAD) {
        total = share ? p.experts * share * 8 : p.experts * of_expert;
    } else {
        if (threadIdx.x < 3) found[threadIdx.x] = 0;
        all.start(p, shared, [](uint32_t n) { return (n + BM - 1) / BM; });
        total = all.total * p.col_tiles;
    }
    for (uint32_t i = blockIdx.x; i / 8 < (total + 7) / 8; i += gridDim.x) {
        uint32_t tile = i;
        if (!(GRAD && share) && !tile_of(i, total, tile)) continue;
        uint32_t e, m0, n0, items, length;   // expert; first row, column; rows; of k
        const char *from, *col_from;
        if constexpr (GRAD) {
            e = share ? tile / 8 / share : tile / of_expert;
            const uint32_t rest = share ? tile % 8 * share + tile / 8 % share : tile % of_expert;
            if (rest >= of_expert) continue;
            m0 = rest % p.row_tiles * BM;
            n0 = rest / p.row_tiles * BN;
            uint32_t lo, hi;
            expert_rows(p, e, lo, hi);
            length = hi - lo;
            items = p.m - m0;
            from = p.row + lo * p.row_stride + (uint64_t)m0 * P::kSize;
            col_from = p.col + lo * p.col_stride + (uint64_t)n0 * P::kSize;
        } else {
            // groups of four row tiles, column by column
            const uint32_t group = tile / (4 * p.col_tiles), rest = tile - group * 4 * p.col_tiles;
            const uint32_t left = all.total - group * 4, high = left < 4 ? left : 4;
            all.find(group * 4 + rest % high, BM, found);
            e = found[0];
            m0 = found[1];
            items = found[2] - m0;
            if (items == 0) continue;
            n0 = rest / high * BN;
            length = p.k * P::kSize;
            from = p.row + m0 * p.row_stride;
            col_from = p.col + e * p.col_expert + n0 * (ACROSS ? (uint64_t)P::kSize : p.col_stride);
        }
        Rows rows;
        Columns columns;
        // across operands count k in rows
        const uint32_t col_length = ACROSS && !GRAD ? p.k : length;
        rows.start(from, p.row_stride, items, length);
        columns.start(col_from, p.col_stride, p.n - n0, col_length);
        f32x16 acc[RB][CB], late[RB][CB];   // HALVES: of the second half in late
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int c = 0; c < CB; ++c) acc[r][c] = late[r][c] = f32x16{};

        const uint32_t per = GRAD ? Rows::kRows : 128;
        const uint32_t steps = (length + per - 1) / per;
        // where this lane's rows and columns have their scales
        const char *rs[RB], *cs[CB];
        if constexpr (__is_same(P, PE4M3) || __is_same(P, PMx4)) {
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                const uint32_t row = (wr * RB + r) * 32 + l % 32;
                rs[r] = p.row_scale + (m0 + (row < items ? row : items - 1)) * p.row_scale_stride;
            }
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                uint32_t col = n0 + (wc * CB + c) * 32 + (__is_same(P, PMx4) ? l % 32 : 0);
                col = col < p.n ? col : p.n - 1;
                cs[c] = p.col_scale + e * p.col_scale_expert +
                        (__is_same(P, PMx4) ? col : col / 128) * p.col_scale_stride;
            }
        }
        auto multiply_step = [&](uint32_t t, lds_bytes row_step, lds_bytes column_step) {
            if constexpr (__is_same(P, PE4M3)) {
                u32x4 rf[4][RB], cf[4][CB];
#pragma unroll
                for (int s = 0; s < 4; ++s) {
#pragma unroll
                    for (int r = 0; r < RB; ++r) rf[s][r] = Rows::fragment(row_step, wr * RB + r, s);
#pragma unroll
                    for (int c = 0; c < CB; ++c)
                        cf[s][c] = Columns::fragment(column_step, wc * CB + c, s);
                }
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const float a = *(const float *)(rs[r] + t * 4ull);
#pragma unroll
                    for (int c = 0; c < CB; ++c) {
                        const float by = a * *(const float *)(cs[c] + t * 4ull);
                        f32x16 part = multiply_e4m3(cf[0][c], cf[1][c], rf[0][r], rf[1][r], f32x16{});
                        if constexpr (HALVES) {
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                acc[r][c][j] = __builtin_fmaf(part[j], by, acc[r][c][j]);
                            part = f32x16{};
                        }
                        part = multiply_e4m3(cf[2][c], cf[3][c], rf[2][r], rf[3][r], part);
                        f32x16 &to = HALVES ? late[r][c] : acc[r][c];
#pragma unroll
                        for (int j = 0; j < 16; ++j) to[j] = __builtin_fmaf(part[j], by, to[j]);
                    }
                }
            } else {
                uint32_t re[RB], ce[CB];   // mx4: four exponents each
                if constexpr (__is_same(P, PMx4)) {
                    const uint32_t at = t * 8 + 4 * h, count = p.k / 16;
                    auto exponents = [&](const char *from) {
                        if (at + 4 <= count)
                            return *(const __attribute__((address_space(1))) u32_any *)((global_bytes)from + at);
                        uint32_t v = 0;
#pragma unroll
                        for (uint32_t j = 0; j < 4; ++j)
                            if (at + j < count) v |= (uint32_t)(uint8_t)from[at + j] << (8 * j);
                        return v;
                    };
#pragma unroll
                    for (int r = 0; r < RB; ++r) re[r] = exponents(rs[r]);
#pragma unroll
                    for (int c = 0; c < CB; ++c) ce[c] = exponents(cs[c]);
                }
                auto sub_step = [&](auto sub) {
                    constexpr int S = decltype(sub)::value;
                    u32x4 rf[RB], cf[CB];
#pragma unroll
                    for (int r = 0; r < RB; ++r) rf[r] = Rows::fragment(row_step, wr * RB + r, S);
#pragma unroll
                    for (int c = 0; c < CB; ++c) cf[c] = Columns::fragment(column_step, wc * CB + c, S);
#pragma unroll
                    for (int r = 0; r < RB; ++r)
#pragma unroll
                        for (int c = 0; c < CB; ++c) {
                            f32x16 &to = HALVES && S >= 2 ? late[r][c] : acc[r][c];
                            if constexpr (__is_same(P, PMx4))
                                to = multiply_mx4<S>(cf[c], rf[r], ce[c], re[r], to);
                            else
                                to = multiply<P>(cf[c], rf[r], to);
                        }
                };
                sub_step(std::integral_constant<int, 0>{});
                sub_step(std::integral_constant<int, 1>{});
                sub_step(std::integral_constant<int, 2>{});
                sub_step(std::integral_constant<int, 3>{});
            }
        };
        const lds_bytes r0 = (lds_bytes)rows0, r1 = (lds_bytes)rows1;
        const lds_bytes c0 = (lds_bytes)columns0, c1 = (lds_bytes)columns1;
        // a step's loads are on their way while the step before is multiplied
        auto step = [&](uint32_t t, lds_bytes rn, lds_bytes cn, lds_bytes rt, lds_bytes ct) {
            if (t + 1 < steps) {
                rows.load(t + 1, length, rn);
                columns.load(t + 1, col_length, cn);
            }
            multiply_step(t, rt, ct);
            if (t + 1 < steps) {
                rows.store(t + 1, length, rn);
                columns.store(t + 1, col_length, cn);
            }
            __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
        };
        if (steps) {
            rows.load(0, length, r0);
            columns.load(0, col_length, c0);
            rows.store(0, length, r0);
            columns.store(0, col_length, c0);
            __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            for (uint32_t t = 0; t < steps; t += 2) {
                step(t, r1, c1, r0, c0);
                if (t + 1 < steps) step(t + 1, r0, c0, r1, c1);
            }
        }
        if constexpr (HALVES)
#pragma unroll
            for (int r = 0; r < RB; ++r)
#pragma unroll
                for (int c = 0; c < CB; ++c) acc[r][c] += late[r][c];
        char *out = p.out + (GRAD ? e * p.out_expert : 0) + m0 * p.out_stride;
        auto leave = [&](uint32_t row, uint32_t col, float (&v)[4]) {
            if (row >= items || col >= p.n) return;
            char *to = out + row * p.out_stride;
            const uint32_t n = p.n - col < 4 ? p.n - col : 4;
            if (GRAD && p.add)
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j)
                    if (j < n) v[j] += value_at(to, col + j, p.out_type);
            store_four(to, col, n, v, p.out_type);
        };
        // Results of the larger tiles leave through LDS, a wave's 32 x 32 at a time in a part of
        // the first step's buffer, so that a store has 8 lanes' 4 columns of a row side by side
        // and not 2 (gradient of 4097 x 2049 bf16, 32768 rows: 1745 to 1540 us; the smaller ones
        // and e4m3, short of registers, lose 5 to 10 % by it).  A wave's accesses to LDS happen
        // in order.
        constexpr bool STAGED = RB == 2 && !__is_same(P, PE4M3);
        const lds_bytes stage = r0 + wave * 4096;
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
            for (int c = 0; c < CB; ++c) {
                const uint32_t row0 = (wr * RB + r) * 32, col0 = n0 + (wc * CB + c) * 32;
                if constexpr (STAGED) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *(__attribute__((address_space(3))) u32x4 *)(
                            stage + l % 32 * 128 + ((2 * q + h) ^ l % 8) * 16) =
                            u32x4{__float_as_uint(acc[r][c][4 * q]), __float_as_uint(acc[r][c][4 * q + 1]),
                                  __float_as_uint(acc[r][c][4 * q + 2]), __float_as_uint(acc[r][c][4 * q + 3])};
                    __builtin_amdgcn_wave_barrier();
                }
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q) {
                    float v[4];
                    if constexpr (STAGED) {
                        const uint32_t row = q * 8 + l / 8;
                        const u32x4 x = *(const __attribute__((address_space(3))) u32x4 *)(
                            stage + row * 128 + (l % 8 ^ row % 8) * 16);
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(x[j]);
                        leave(row0 + row, col0 + l % 8 * 4, v);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] = acc[r][c][4 * q + j];
                        leave(row0 + l % 32, col0 + 8 * q + 4 * h, v);
                    }
                }
                if constexpr (STAGED) __builtin_amdgcn_wave_barrier();
            }
        if constexpr (STAGED) __syncthreads();   // the next tile's first step goes there
    }
}

template <class P, bool GRAD, bool ACROSS, bool DIRECT, int RB, int CB, bool HALVES = false>
hipError_t go_product(ProductParams p, hipStream_t s)
{
    constexpr uint32_t BM = 64 * RB, BN = 64 * CB;
    p.col_tiles = (p.n + BN - 1) / BN;
    p.row_tiles = (p.m + BM - 1) / BM;
    // forward: every expert may end in a tile that is not whole
    const uint64_t tiles = GRAD ? (uint64_t)p.experts * p.row_tiles
                                : p.rows / BM + (p.rows < p.experts ? p.rows : p.experts);
    p.most = (uint32_t)tiles;
    return launch_kernel(product_kernel<P, GRAD, ACROSS, DIRECT, RB, CB, HALVES>,
                         dim3(grid_of((tiles * p.col_tiles + 7) / 8 * 8, kProductThreads)),
                         dim3(kProductThreads), 0, s, p);
}

// Whether an operand's 16-byte pieces lie on the 16-byte grid, whole ones only, so that
// loads can go straight to LDS.
inline bool on_grid(const char *base, uint64_t stride, uint64_t apart, uint64_t width)
{
    return ((uintptr_t)base | stride | apart | width) % 16 == 0;
}

}  // namespace xred
