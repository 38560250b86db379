// Attention of trees of drafted tokens to a paged key/value cache: the kernels of attention_launch.h with an ancestor mask.
//
// A row of a tree sees what is cached before the tree, and of the tree's own rows those whose bits its mask has.  Only the steps that reach past
// the cached tokens ask for the masks: 64 bits of them, put together from two words, hold what a row sees of a step's tokens.
//
// The kernels are of their own, so that those without trees keep their code.  What bounds them is what bounds those: 32 trees of 16 to 64 rows, 32 heads over 8, over up to 8192
// tokens 135 to 140 us by card (389 MB, and again where a tree has more than 128 packed rows: 2.8 TB/s; matrix pipes 20 % busy, a quarter of their rows padding); one of 26
// rows over 700 tokens 20.5 us, 16 blocks of a plan, six steps and a join of pieces, each a few us.  The kernel of few rows keeps 7 registers in scratch at 128 dimensions in bf16.
#include "attention_launch.h"

namespace moe {

hipError_t launch_tree_attention(int dtype, bool fp8, const AttnArgs& a, bool clear, hipStream_t s)
{
    return launch_by_type<true>(dtype, fp8, a, clear, s);
}

}  // namespace moe
