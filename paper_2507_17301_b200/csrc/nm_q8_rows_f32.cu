#include "nm_q8_rows.cuh"

namespace nmhost {
nm_status_t launch_q8_rows_f32(Q8RowOp op, const Q8Rows& a, nm_dtype_t weight_type, bool vec, cudaStream_t st)
{
    return q8rows::launch<float>(op, a, weight_type, vec, st);
}
}  // namespace nmhost
