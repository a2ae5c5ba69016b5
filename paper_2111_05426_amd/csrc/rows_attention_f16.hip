// rows_attention_f16.hip -- the kernels of prompt and tree attention for fp16 queries.
#include "rows_attention.h"

namespace dsim {
namespace rows {

dsim_status launch_f16(Params &p, bool e4m3_cache, hipStream_t s)
{
    return e4m3_cache ? launch<f16, e4m3>(p, s) : launch<f16, f16>(p, s);
}

}  // namespace rows
}  // namespace dsim
