// The instances of the paged attention kernel for keys of 3 bits.
#include "attention_paged.cuh"
#include "attention_paged_launch.h"

namespace rptq {
namespace attn_paged {

int launch_keys3(const Params& p, const Launch& l) { return launch_values<3>(p, l); }

}  // namespace attn_paged
}  // namespace rptq
