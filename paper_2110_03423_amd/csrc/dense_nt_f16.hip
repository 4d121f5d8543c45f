#include "dense_nt.hpp"

namespace rsvd {
DENSE_NT(DK_F16, true)
}  // namespace rsvd
