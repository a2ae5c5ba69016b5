// rows_attention_f32.hip -- the kernels of prompt and tree attention for fp32 queries.
#include "rows_attention.h"

namespace dsim {
namespace rows {

dsim_status launch_f32(Params &p, hipStream_t s)
{
    return launch<float, float>(p, s);
}

}  // namespace rows
}  // namespace dsim
