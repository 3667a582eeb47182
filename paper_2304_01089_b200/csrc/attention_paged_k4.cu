// The instances of the paged attention kernel for keys of 4 bits.
#include "attention_paged.cuh"
#include "attention_paged_launch.h"

namespace rptq {
namespace attn_paged {

int launch_keys4(const Params& p, const Launch& l) { return launch_values<4>(p, l); }

}  // namespace attn_paged
}  // namespace rptq
