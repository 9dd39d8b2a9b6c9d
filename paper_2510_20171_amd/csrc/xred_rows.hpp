// xred_rows.hpp -- device helpers shared by the kernels that work on rows
// (norm, dispatch, combine): pieces of 8 elements at any element alignment,
// and reductions over a wave and a workgroup.
//
// A row is cut into pieces of 8 elements; a lane owns whole pieces, so a lane
// moves 16 bytes of a 2-byte type (32 of fp32, 8 of e4m3) at a time.  Rows may
// start at any element, so pieces are read and written with unaligned global
// accesses, which cost no more than aligned ones where rows are aligned.  Only
// a row's last piece may be short; one lane moves it element by element.
#pragma once

#include <type_traits>

#include "xred_kernels.hpp"

namespace xred {

typedef __attribute__((address_space(1))) char *global_out;

// 8 consecutive elements as they lie in memory.
template <class T>
struct Piece {
    static constexpr int kWords = T::kSize * 8 / 16;
    u32x4 w[kWords];
};

// off: bytes from base, the same base in every lane.  KEEP: the data is read
// again soon (by other workgroups), else it is streamed.
template <class T, bool KEEP = false>
__device__ __forceinline__ Piece<T> load_piece(const char *base, uint32_t off)
{
    Piece<T> r;
#pragma unroll
    for (int i = 0; i < Piece<T>::kWords; ++i) {
        const auto *p =
            (const __attribute__((address_space(1))) u32x4_any *)((global_bytes)base + off + 16 * i);
        r.w[i] = KEEP ? *p : __builtin_nontemporal_load(p);
    }
    return r;
}

template <class T>
__device__ __forceinline__ void up_piece(const Piece<T> &r, float (&a)[8])
{
#pragma unroll
    for (int i = 0; i < Piece<T>::kWords; ++i) {
        float b[T::kVec];
        up_vec<T>(r.w[i], b);
#pragma unroll
        for (int j = 0; j < T::kVec; ++j) a[i * T::kVec + j] = b[j];
    }
}

// The same values, hidden from the optimiser.
template <class T>
__device__ __forceinline__ void opaque_piece(Piece<T> &r)
{
#pragma unroll
    for (int i = 0; i < Piece<T>::kWords; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t x = r.w[i][j];
            __asm__ volatile("" : "+v"(x));
            r.w[i][j] = x;
        }
}

// The first c elements of a row's last piece (c < 8, at byte `off`); 0 past them.
template <class T>
__device__ __forceinline__ void up_short(const char *base, uint32_t off, uint32_t c, float (&a)[8])
{
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) a[j] = j < c ? up1<T>(base + off, j) : 0.0f;
}

// The same as it lies in memory.
template <class T>
__device__ __forceinline__ Piece<T> short_piece(const char *base, uint32_t off, uint32_t c)
{
    using Bits = std::conditional_t<T::kSize == 4, uint32_t, uint16_t>;
    constexpr uint32_t kPer = 4 / T::kSize;   // elements of a dword
    Piece<T> r;
#pragma unroll
    for (uint32_t i = 0; i < 8 / kPer; ++i) {
        uint32_t x = 0;
#pragma unroll
        for (uint32_t j = 0; j < kPer; ++j)
            if (i * kPer + j < c)
                x |= (uint32_t)((const Bits *)(base + off))[i * kPer + j] << (16 * j);
        r.w[i / 4][i % 4] = x;
    }
    return r;
}

// Elements of piece i that exist: 8, fewer at the end of the row, 0 past it.
__device__ __forceinline__ uint32_t piece_count(uint32_t i, uint32_t n)
{
    const uint32_t at = 8 * i;
    return at >= n ? 0u : n - at < 8 ? n - at : 8u;
}

template <class T>
__device__ __forceinline__ void store_piece(char *base, uint32_t off, uint32_t c,
                                            const float (&a)[8])
{
    if (c == 8) {
#pragma unroll
        for (int i = 0; i < Piece<T>::kWords; ++i) {
            float b[T::kVec];
#pragma unroll
            for (int j = 0; j < T::kVec; ++j) b[j] = a[i * T::kVec + j];
            *(__attribute__((address_space(1))) u32x4_any *)((global_out)base + off + 16 * i) =
                down_vec<T, OpSum>(b);
        }
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
            if (j < c) down1<T, OpSum>(base + off, j, a[j]);
    }
}

// The same for e4m3 (8 bytes a piece).
__device__ __forceinline__ void store_piece_e4m3(char *base, uint32_t off, uint32_t c,
                                                 const float (&a)[8])
{
    u32x2 q;
    q[0] = pack_fp8x4<TE4M3>(a[0], a[1], a[2], a[3]);
    q[1] = pack_fp8x4<TE4M3>(a[4], a[5], a[6], a[7]);
    if (c == 8) {
        *(__attribute__((address_space(1))) u32x2_any *)((global_out)base + off) = q;
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
            if (j < c) base[off + j] = (char)(q[j / 4] >> (8 * (j % 4)));
    }
}

// ------------------------------------------------------------- reductions --
// x of the lane l ^ M, as seen by lane l (M a power of two below 64; every lane
// of the wave takes part).
template <int M, class X>
__device__ __forceinline__ X lane_xor(X x)
{
    static_assert(sizeof(X) == 4, "one register");
    const int v = __builtin_bit_cast(int, x);
    int r;
    if constexpr (M == 1) r = __builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true);        // quad 1 0 3 2
    else if constexpr (M == 2) r = __builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true);   // quad 2 3 0 1
    else if constexpr (M == 8) r = __builtin_amdgcn_mov_dpp(v, 0x128, 0xF, 0xF, true);  // row_ror 8
    else if constexpr (M == 16 || M == 4) r = __builtin_amdgcn_ds_swizzle(v, (M << 10) | 0x1F);
    else r = __shfl_xor(v, 32);
    return __builtin_bit_cast(X, r);
}

// A sum and a maximum (NaN-propagating, like every maximum here) over aligned
// sets of N lanes; every lane has the result.  The order of the additions is
// fixed by the lanes' places.
template <int N, int M = 1>
__device__ __forceinline__ float lanes_sum(float x)
{
    if constexpr (M < N) return lanes_sum<N, 2 * M>(x + lane_xor<M>(x));
    else return x;
}

template <int N, int M = 1>
__device__ __forceinline__ float lanes_max(float x)
{
    if constexpr (M < N)
        return lanes_max<N, 2 * M>(__builtin_elementwise_maximum(x, lane_xor<M>(x)));
    else return x;
}

template <int N, int M = 1>
__device__ __forceinline__ int lanes_max(int x)
{
    if constexpr (M < N) {
        const int y = lane_xor<M>(x);
        return lanes_max<N, 2 * M>(x > y ? x : y);
    } else {
        return x;
    }
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
