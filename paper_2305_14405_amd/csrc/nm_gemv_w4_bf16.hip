// nm_gemv_w4: its kernels for bf16 rows (nm_gemv_w4.h).
#include "nm_gemv_w4.h"

namespace nm {
template int32_t launch_w4<bf16>(const W4Args&, hipStream_t);
}  // namespace nm
