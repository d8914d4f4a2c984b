#define S2A_ROPE_WHOLE_ROWS
#include "s2a_rope.cuh"

namespace s2a {
template cudaError_t launch_rope_whole<kBF16>(int, const RopeArgs&, unsigned, cudaStream_t);
}
