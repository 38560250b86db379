// Attention of a batch's rows, as they follow each other, to a paged key/value cache: attention_launch.h.
#include "attention_launch.h"

namespace moe {

hipError_t launch_attention(int dtype, bool fp8, const AttnArgs& a, bool clear, hipStream_t s)
{
    return launch_by_type<false>(dtype, fp8, a, clear, s);
}

}  // namespace moe
