// Attention kernels of f32 rows.
#include "attention.hpp"

namespace sn {
namespace k {

void attention_f32(AttnArgs& a, bool step, hipStream_t st) { launch_attention<float>(a, step, st); }

}  // namespace k
}  // namespace sn
