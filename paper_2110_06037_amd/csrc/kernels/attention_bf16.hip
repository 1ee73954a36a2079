// Attention kernels of bf16 rows.
#include "attention.hpp"

namespace sn {
namespace k {

void attention_bf16(AttnArgs& a, bool step, hipStream_t st) { launch_attention<bf16>(a, step, st); }

}  // namespace k
}  // namespace sn
