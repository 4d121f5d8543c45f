#include "dense_nt.hpp"

namespace rsvd {
DENSE_NT(DK_F16, false)
}  // namespace rsvd
