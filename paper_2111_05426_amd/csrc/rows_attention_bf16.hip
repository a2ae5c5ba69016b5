// rows_attention_bf16.hip -- the kernels of prompt and tree attention for bf16 queries.
#include "rows_attention.h"

namespace dsim {
namespace rows {

dsim_status launch_bf16(Params &p, bool e4m3_cache, hipStream_t s)
{
    return e4m3_cache ? launch<bf16, e4m3>(p, s) : launch<bf16, bf16>(p, s);
}

}  // namespace rows
}  // namespace dsim
