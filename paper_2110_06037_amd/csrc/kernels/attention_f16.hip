// Attention kernels of f16 rows.
#include "attention.hpp"

namespace sn {
namespace k {

void attention_f16(AttnArgs& a, bool step, hipStream_t st) { launch_attention<f16>(a, step, st); }

}  // namespace k
}  // namespace sn
