// xred_product_launch.hpp -- launchers of the experts' products, one translation
// unit for each operand type.  Arguments were validated by the caller.
#pragma once

#include "xred_layer.hpp"

namespace xred {

// A product as the kernels see it (xred_product.hpp): operands of the output's rows and
// columns; distances and offsets in bytes.
struct ProductParams {
    const char *row, *col;
    const char *row_scale, *col_scale;
    char *out;
    const int32_t *offsets;
    uint64_t row_stride, col_stride, out_stride;   // from row to row
    uint64_t col_expert, out_expert;               // from expert to expert
    uint64_t row_scale_stride, col_scale_stride, col_scale_expert;
    uint32_t rows;      // of x
    uint32_t m, n;      // the output's rows (gradient: of one expert) and columns
    uint32_t k;         // forward: elements summed over (mx4: bytes, two elements each)
    uint32_t experts;
    uint32_t row_tiles, col_tiles;   // set by the launcher
    uint32_t most;                   // the same: what RowTiles counts, at most, of offsets that ascend
    uint32_t spans;                  // the same: several columns of an expert's last rows in one
    xred_dtype out_type;
    uint32_t add;
};

hipError_t launch_product_bf16(const ProductParams &p, bool grad, bool across, hipStream_t s);
hipError_t launch_product_f16(const ProductParams &p, bool grad, bool across, hipStream_t s);
hipError_t launch_product_f32(const ProductParams &p, bool grad, bool across, hipStream_t s);
hipError_t launch_product_e4m3(const ProductParams &p, hipStream_t s);
hipError_t launch_product_mx4(const ProductParams &p, hipStream_t s);

}  // namespace xred
