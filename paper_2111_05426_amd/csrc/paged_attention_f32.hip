// paged_attention_f32.hip -- the kernels of dsim_paged_attention for fp32 queries.
#include "paged_attention.h"

namespace dsim {
namespace attend {

dsim_status launch_f32(Params &p, hipStream_t s) { return launch<float, float>(p, s); }

}  // namespace attend
}  // namespace dsim
