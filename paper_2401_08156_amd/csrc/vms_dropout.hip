// vms_dropout (include/vms_ops.h): residual + dropout(x), forward and backward alike.
#include "ops_common.hpp"

namespace {

struct DropoutParams {
    const void *x, *residual;
    void *y;
    u64 ldx, ldr, ldy;
    u64 groups;                 // of eight columns, over all rows
    u32 rows, cols, per_row;    // groups of a row
    Mask mask;
};

// A lane takes groups of eight consecutive elements of a row, `step` groups apart.  Their row and place in it are found by
// one division and carried on by additions.
template <class T, bool ONCE>
__global__ __launch_bounds__(256) void dropout_kernel(const DropoutParams p)
{
    const u64 seed = p.mask.limit ? mask_seed(p.mask) : 0;
    const u64 step = (u64)gridDim.x * 256;
    u64 at = (u64)blockIdx.x * 256 + threadIdx.x;
    const u32 step_rows = (u32)(step / p.per_row), step_groups = (u32)(step % p.per_row);
    u32 row = (u32)(at / p.per_row), group = (u32)(at % p.per_row);
    for (; at < p.groups; at += step) {
        const u32 col = group * 8, n = p.cols - col;
        float v[8];
        load8<ONCE>((const T *)p.x + row * p.ldx + col, n, v);
        float r[8];
        if (p.residual) load8<ONCE>((const T *)p.residual + row * p.ldr + col, n, r);
        if (p.mask.limit) drop8(p.mask, seed, row, group, v);
        if (p.residual) {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] += r[i];
        }
        store8<ONCE>((T *)p.y + row * p.ldy + col, n, v);
        row += step_rows;
        group += step_groups;
        if (group >= p.per_row) {
            group -= p.per_row;
            row++;
        }
    }
}

}  // namespace

extern "C" int vms_dropout(const vms_dropout_args *a, void *stream)
{
    if (!a) return VMS_EINVAL;
    if (a->struct_size != sizeof *a) return VMS_ESTRUCT;
    DropoutParams p;
    int rc = make_mask(a->mask, &p.mask);
    if (rc) return rc;
    if (a->dtype > VMS_BF16 || a->rows >> 31 || a->cols >> 31) return VMS_EINVAL;
    if (!a->rows || !a->cols) return VMS_OK;
    if (!input_ok(a->d_x, a->dtype) || !output_ok(a->d_y, a->dtype, a->ldy, a->cols)) return VMS_EINVAL;
    if (a->d_residual && !input_ok(a->d_residual, a->dtype)) return VMS_EINVAL;
    if (!stride_ok(a->ldx) || !stride_ok(a->ldr) || !stride_ok(a->ldy)) return VMS_EINVAL;
    p.x = a->d_x;
    p.residual = a->d_residual;
    p.y = a->d_y;
    p.ldx = a->ldx;
    p.ldr = a->ldr;
    p.ldy = a->ldy;
    p.rows = (u32)a->rows;
    p.cols = (u32)a->cols;
    p.per_row = (p.cols + 7) / 8;
    p.groups = (u64)p.rows * p.per_row;
    const u64 blocks = (p.groups + 255) / 256;
    const u32 grid = (u32)(blocks < OPS_CUS * 32 ? blocks : OPS_CUS * 32);
    const bool once = passes_by(a->rows * a->cols * type_bytes(a->dtype) * (a->d_residual ? 3 : 2));
    return with_type(a->dtype, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        return ops_launch(once ? dropout_kernel<T, true> : dropout_kernel<T, false>, dim3(grid), dim3(256), 0, p, stream);
    });
}
