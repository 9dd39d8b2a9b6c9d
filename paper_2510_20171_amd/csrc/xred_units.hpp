// xred_units.hpp -- rows cut into units of 8 elements, a lane each, for the kernels
// that work on every element of a row by itself or with its neighbours (gated
// activation, 4-bit quantisation).
//
// A unit is one 16-byte vector of a 2-byte type, two of fp32.  Rows lie at any
// element; only a row's last unit may be short, and is read as the row's last 8
// elements, shifted into place.  An item is up to 64 units of one row, which as many
// lanes work on (a power of two); a wave takes 64 / lanes items at a time.
#pragma once

#include "xred_layer.hpp"
#include "xred_rows.hpp"

namespace xred {

constexpr int kUnitThreads = 256;

struct UnitItems {
    uint32_t items, per_row;   // in all; of a row
    uint32_t lanes;            // of an item
};

// Items of `rows` rows of n elements (fewer items than 2^32, as the caller checked), in units
// of UNIT, and the grid that takes them.  32 elements are never split between items.
template <int UNIT = 8>
unsigned plan_units(uint64_t rows, uint64_t n, UnitItems &u)
{
    const uint64_t units = (n + UNIT - 1) / UNIT, per_row = (units + 63) / 64;
    u.lanes = 64;
    while (u.lanes > 32 / UNIT && u.lanes / 2 >= units) u.lanes /= 2;
    u.items = (uint32_t)(rows * per_row);
    u.per_row = (uint32_t)per_row;
    const uint64_t at_once = kUnitThreads / u.lanes;
    return grid_of((u.items + at_once - 1) / at_once, kUnitThreads);
}

// Item i's row and this lane's unit of it.
__device__ __forceinline__ void unit_of(const UnitItems &u, uint64_t i, uint32_t &row, uint32_t &unit)
{
    const uint32_t lane = threadIdx.x % u.lanes;
    if (u.per_row == 1) {
        row = (uint32_t)i;
        unit = lane;
    } else {   // a wave's item
        const uint32_t item = __builtin_amdgcn_readfirstlane((uint32_t)i);
        row = item / u.per_row;
        unit = item % u.per_row * 64 + lane;
    }
}

// The raw vectors of a unit, on their way.
template <class T>
struct UnitRaw {
    static constexpr int kVecs = 8 / T::kVec;
    u32x4 v[kVecs];
    // n >= 8; c: elements of the unit (0: past the row's end)
    __device__ __forceinline__ void load(const char *row, uint32_t unit, uint32_t c, uint32_t n)
    {
        const uint32_t from = (c == 8 ? unit * 8 : n - 8) * T::kSize;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i] = load_piece(row, from + 16 * i);
    }
    __device__ __forceinline__ void up(float (&x)[8], uint32_t c, uint32_t n) const
    {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            float y[T::kVec];
            up_vec<T>(v[i], y);
#pragma unroll
            for (int j = 0; j < T::kVec; ++j) x[i * T::kVec + j] = y[j];
        }
        settle<8>(x, c, n);
    }
};

// A unit of a row shorter than one.
template <class T>
__device__ __forceinline__ void up_short_unit(const char *row, uint32_t c, float (&x)[8])
{
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) x[j] = j < c ? up1<T>(row, j) : 0.0f;
}

template <class T>
__device__ __forceinline__ void store_unit(char *row, uint32_t unit, uint32_t c, const float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < UnitRaw<T>::kVecs; ++i) {
        float y[T::kVec];
#pragma unroll
        for (int j = 0; j < T::kVec; ++j) y[j] = x[i * T::kVec + j];
        const uint32_t skip = i * T::kVec;
        store_piece<T>(row, unit * 8 * T::kSize + 16 * i,
                       c <= skip ? 0 : c - skip < T::kVec ? c - skip : T::kVec, y);
    }
}

}  // namespace xred
