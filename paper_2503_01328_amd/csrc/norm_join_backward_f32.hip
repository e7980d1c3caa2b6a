// norm_join_backward.h for f32.
#include "norm_join_backward.h"

namespace po {
namespace norm_join {

void launch_backward_f32(const Join& p, hipStream_t stream) { launch_backward<float>(p, stream); }

}  // namespace norm_join
}  // namespace po
