// Attention of trees of drafted tokens to a paged key/value cache: the kernels of attention_launch.h with an ancestor mask.
//
// A row of a tree sees what is cached before the tree, and of the tree's own rows those whose bits its mask has.  Only the steps that reach past
// the cached tokens ask for the masks: 64 bits of them, put together from two words, hold what a row sees of a step's tokens.
#include "attention_launch.h"

namespace moe {

hipError_t launch_tree_attention(int dtype, bool fp8, const AttnArgs& a, bool clear, hipStream_t s)
{
    return launch_by_type<true>(dtype, fp8, a, clear, s);
}

}  // namespace moe
