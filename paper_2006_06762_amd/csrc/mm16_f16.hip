// mm16_kernel.h for f16.
#include "mm16_launch.h"

namespace anr {
namespace mm16 {

hipError_t launch_products_f16(Form form, Shape shape, bool aligned, const Args& a, hipStream_t stream) { return launch_products<half_t>(form, shape, aligned, a, stream); }

}  // namespace mm16
}  // namespace anr
