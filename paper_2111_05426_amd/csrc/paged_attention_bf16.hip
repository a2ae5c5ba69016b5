// paged_attention_bf16.hip -- the kernels of dsim_paged_attention for bf16 queries.
#include "paged_attention.h"

namespace dsim {
namespace attend {

dsim_status launch_bf16(Params &p, bool e4m3_cache, hipStream_t s)
{
    return e4m3_cache ? launch<bf16, e4m3>(p, s) : launch<bf16, bf16>(p, s);
}

}  // namespace attend
}  // namespace dsim
