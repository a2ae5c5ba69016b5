// paged_attention_f16.hip -- the kernels of dsim_paged_attention for fp16 queries.
#include "paged_attention.h"

namespace dsim {
namespace attend {

dsim_status launch_f16(Params &p, bool e4m3_cache, hipStream_t s)
{
    return e4m3_cache ? launch<f16, e4m3>(p, s) : launch<f16, f16>(p, s);
}

}  // namespace attend
}  // namespace dsim
