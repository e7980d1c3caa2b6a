// norm_join_backward.h for bf16.
#include "norm_join_backward.h"

namespace po {
namespace norm_join {

void launch_backward_bf16(const Join& p, hipStream_t stream) { launch_backward<bf16>(p, stream); }

}  // namespace norm_join
}  // namespace po
