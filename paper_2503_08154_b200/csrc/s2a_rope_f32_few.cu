#include "s2a_rope.cuh"

namespace s2a {
template cudaError_t launch_rope_any<kF32, true>(int, uint32_t, uint32_t, const RopeArgs&, unsigned, cudaStream_t);
}
