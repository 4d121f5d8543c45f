#include "dense_kn.hpp"

namespace rsvd {
DENSE_KN(DK_BF16, false)
DENSE_KN(DK_BF16, true)
}  // namespace rsvd
