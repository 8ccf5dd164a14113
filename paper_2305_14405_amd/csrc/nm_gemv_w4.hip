// nm_gemv_w4: the entry point, and its kernels for int8 codes (nm_gemv_w4.h).
#include "nm_gemv_w4.h"

namespace nm {
extern template int32_t launch_w4<bf16>(const W4Args&, hipStream_t);
extern template int32_t launch_w4<f16>(const W4Args&, hipStream_t);
template int32_t launch_w4<int8_t>(const W4Args&, hipStream_t);
}  // namespace nm

using namespace nm;

extern "C" int32_t nm_gemv_w4(const nm_w4_desc* d, void* stream)
{
    if (!d) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: desc is NULL");
    if (d->M < 0 || d->N < 1 || d->K < 1 || d->group < 1) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: bad shape");
    if (d->x_dtype != NM_DT_I8 && d->x_dtype != NM_DT_BF16 && d->x_dtype != NM_DT_F16) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: bad x_dtype");
    if (!float_dtype(d->scale_dtype)) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: bad scale_dtype");
    if (!float_dtype(d->out_dtype) && d->out_dtype != NM_DT_I8) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: bad out_dtype");
    if (d->group != 32 && d->group != 64 && d->group % 128) return fail(NM_ERR_UNSUPPORTED, "nm_gemv_w4: group %d is not 32, 64 or a multiple of 128", d->group);
    if (d->K % d->group) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: K is no multiple of group");
    if (d->K > 65536 || d->M > 1 << 20 || d->N >= 1 << 26) return fail(NM_ERR_UNSUPPORTED, "nm_gemv_w4: K > 65536, M > 2^20 or N >= 2^26");
    if ((((int64_t)d->N + 15) / 16 + 7) / 8 * 8 * ((d->M + 31) / 32) >= 1 << 23) return fail(NM_ERR_UNSUPPORTED, "nm_gemv_w4: N / 16 times M / 32 >= 2^23");
    if (d->x_stride < d->K || d->out_stride < d->N) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: a stride is shorter than a row");
    if (!(d->alpha == d->alpha) || __builtin_isinf(d->alpha)) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: alpha must be finite");
    W4Args a{};
    a.d = *d;
    if (d->table_idx >= 0) {
        const int32_t rc = get_dev_table(d->tables, d->table_idx, &a.table, "nm_gemv_w4");
        if (rc) return rc;
    }
    if (d->M == 0) return NM_OK;   // empty tensors may be NULL pointers
    if (!d->x || !d->W || !d->scales || !d->out) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: NULL argument");
    if (begins_as(d->out, {d->x, d->W, d->scales, d->bias})) return fail(NM_ERR_INVALID_ARG, "nm_gemv_w4: out is an input");
    if (!aligned_rows(d->x, d->x_stride, d->x_dtype, 16 / dtype_bytes(d->x_dtype)) || !aligned(d->W, 16))
        return fail(NM_ERR_UNSUPPORTED, "nm_gemv_w4: x, its rows and W must be 16-byte aligned");
    a.per = fast_div(d->group >= 128 ? d->group / 128 : 1);
    if (d->x_dtype == NM_DT_I8) return nm::launch_w4<int8_t>(a, (hipStream_t)stream);
    if (d->x_dtype == NM_DT_BF16) return nm::launch_w4<bf16>(a, (hipStream_t)stream);
    return nm::launch_w4<f16>(a, (hipStream_t)stream);
}
