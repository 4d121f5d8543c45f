#include "dense_kn.hpp"

namespace rsvd {
DENSE_KN(DK_F16, false)
DENSE_KN(DK_F16, true)
}  // namespace rsvd
