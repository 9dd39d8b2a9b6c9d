// xred_rows.hpp -- device helpers shared by the kernels that work on rows
// (norm, dispatch, combine): pieces of 16 bytes at any element alignment, and
// reductions over a wave and a workgroup.
//
// A row is cut into pieces of one 16-byte vector, N = 8 elements of a 2-byte type
// or 4 of fp32; a lane owns whole pieces, and neighbouring lanes neighbouring
// pieces.  Rows may start at any element, so pieces are read and written with
// unaligned global accesses, which cost no more than aligned ones where rows are
// aligned.  Only a row's last piece may be short: its lane reads the row's last N
// elements and shifts them into place, so every load is a whole one, and stores it
// element by element.
#pragma once

#include "xred_kernels.hpp"

namespace xred {

typedef __attribute__((address_space(1))) char *global_out;

// off: bytes from base, the same base in every lane.  KEEP: the data is read
// again soon (by other workgroups), else it is streamed.
template <bool KEEP = false>
__device__ __forceinline__ u32x4 load_piece(const char *base, uint32_t off)
{
    const auto *p = (const __attribute__((address_space(1))) u32x4_any *)((global_bytes)base + off);
    return KEEP ? *p : __builtin_nontemporal_load(p);
}

// The same values, hidden from the optimiser.
__device__ __forceinline__ void opaque_piece(u32x4 &r)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t x = r[j];
        __asm__ volatile("" : "+v"(x));
        r[j] = x;
    }
}

// Elements of piece i of a row of n: N, fewer at the end of the row, 0 past it.
template <int N>
__device__ __forceinline__ uint32_t piece_count(uint32_t i, uint32_t n)
{
    const uint32_t at = N * i;
    return at >= n ? 0u : n - at < N ? n - at : (uint32_t)N;
}

// Where a lane with c elements of piece i reads N that exist (of a row of n >= N):
// its piece, or the row's last N for the short last piece (and for no piece).
template <int N>
__device__ __forceinline__ uint32_t piece_from(uint32_t i, uint32_t c, uint32_t n)
{
    return c == N ? N * i : n - N;
}

// What was read there as the piece: a short piece's c elements move to the front,
// with 0 behind them.
template <int N>
__device__ __forceinline__ void settle(float (&x)[N], uint32_t c, uint32_t n)
{
    if (c == N) return;
    if (n % N) {   // the short piece's length, the same for every row
        const uint32_t by = N - n % N;
        if (N == 8 && (by & 4))
#pragma unroll
            for (int j = 0; j < N - 4; ++j) x[j] = x[j + 4];
        if (by & 2)
#pragma unroll
            for (int j = 0; j < N - 2; ++j) x[j] = x[j + 2];
        if (by & 1)
#pragma unroll
            for (int j = 0; j < N - 1; ++j) x[j] = x[j + 1];
    }
#pragma unroll
    for (uint32_t j = 0; j < N; ++j) x[j] = j < c ? x[j] : 0.0f;
}

// The same of a row shorter than a piece, element by element.
template <class T>
__device__ __forceinline__ void up_short(const char *base, uint32_t c, float (&a)[T::kVec])
{
#pragma unroll
    for (uint32_t j = 0; j < T::kVec; ++j) a[j] = j < c ? up1<T>(base, j) : 0.0f;
}

// Outputs are streamed past the caches (nontemporal): beside eight streams that
// are read, ordinary stores cost 140 us where these take 129 (8192 x 4096 bf16).
template <class T>
__device__ __forceinline__ void store_piece(char *base, uint32_t off, uint32_t c,
                                            const float (&a)[T::kVec])
{
    if (c == T::kVec) {
        __builtin_nontemporal_store(
            down_vec<T, OpSum>(a),
            (__attribute__((address_space(1))) u32x4_any *)((global_out)base + off));
    } else {
#pragma unroll
        for (uint32_t j = 0; j < T::kVec; ++j)
            if (j < c) down1<T, OpSum>(base + off, j, a[j]);
    }
}

// The same for e4m3 (a byte an element), values that are at most 448 or NaN: the
// conversion itself gives NaN for more.
template <int N>
__device__ __forceinline__ void store_piece_e4m3(char *base, uint32_t off, uint32_t c,
                                                 const float (&a)[N])
{
    uint32_t q[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a[4 * i], a[4 * i + 1], 0, false);
        q[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a[4 * i + 2], a[4 * i + 3], low, true);
    }
    if (c == N) {
        if constexpr (N == 8)
            __builtin_nontemporal_store(
                u32x2{q[0], q[1]},
                (__attribute__((address_space(1))) u32x2_any *)((global_out)base + off));
        else
            __builtin_nontemporal_store(
                q[0], (__attribute__((address_space(1))) u32_any *)((global_out)base + off));
    } else {
#pragma unroll
        for (uint32_t j = 0; j < N; ++j)
            if (j < c) base[off + j] = (char)(q[j / 4] >> (8 * (j % 4)));
    }
}

// ------------------------------------------------------------- reductions --
// The two halves of aligned sets of 2 * M lanes, each half of M lanes already
// reduced to one value: a holds one half's, b the other's (in either order).  The
// steps up to 16 lanes are data-parallel moves, the last two swap rows of 16 and
// 32 lanes, so a reduction never waits for LDS.  Every lane of the wave takes part.
struct Halves {
    uint32_t a, b;
};
template <int M>
__device__ __forceinline__ Halves halves(uint32_t x)
{
    const int v = (int)x;
    if constexpr (M == 1) {          // quads 1 0 3 2
        return {x, (uint32_t)__builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true)};
    } else if constexpr (M == 2) {   // quads 2 3 0 1
        return {x, (uint32_t)__builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true)};
    } else if constexpr (M == 4) {   // 8 lanes mirrored
        return {x, (uint32_t)__builtin_amdgcn_mov_dpp(v, 0x141, 0xF, 0xF, true)};
    } else if constexpr (M == 8) {   // 16 lanes mirrored
        return {x, (uint32_t)__builtin_amdgcn_mov_dpp(v, 0x140, 0xF, 0xF, true)};
    } else if constexpr (M == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return {r[0], r[1]};
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return {r[0], r[1]};
    }
}

// A sum and maxima (of floats: NaN-propagating, like every maximum here) over
// aligned sets of N lanes; every lane has the result.  The order of the additions
// is fixed by the lanes' places.
template <int N, int M = 1>
__device__ __forceinline__ float lanes_sum(float x)
{
    if constexpr (M < N) {
        const Halves h = halves<M>(__float_as_uint(x));
        return lanes_sum<N, 2 * M>(__uint_as_float(h.a) + __uint_as_float(h.b));
    } else {
        return x;
    }
}

template <int N, int M = 1>
__device__ __forceinline__ float lanes_max(float x)
{
    if constexpr (M < N) {
        const Halves h = halves<M>(__float_as_uint(x));
        return lanes_max<N, 2 * M>(
            __builtin_elementwise_maximum(__uint_as_float(h.a), __uint_as_float(h.b)));
    } else {
        return x;
    }
}

template <int N, int M = 1>
__device__ __forceinline__ int lanes_max(int x)
{
    if constexpr (M < N) {
        const Halves h = halves<M>((uint32_t)x);
        return lanes_max<N, 2 * M>((int)h.a > (int)h.b ? (int)h.a : (int)h.b);
    } else {
        return x;
    }
}

// Sum of x over the lanes below this one in its set of L, and over all of them.
template <int L>
__device__ __forceinline__ void lanes_before(uint32_t x, uint32_t &before, uint32_t &all)
{
    uint32_t s = x;   // row_shr 1, 2, 4, 8; then the rows before
    s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x111, 0xF, 0xF, true);
    s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x112, 0xF, 0xF, true);
    s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x114, 0xF, 0xF, true);
    s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x118, 0xF, 0xF, true);
    if constexpr (L == 64) {
        s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x142, 0xA, 0xF, false);
        s += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x143, 0xC, 0xF, false);
    }
    before = s - x;
    all = (uint32_t)lanes_max<L>((int)s);
}

// Orders a wave's LDS accesses before it against those after it, for lanes that
// read what other lanes of their wave wrote.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

}  // namespace xred
