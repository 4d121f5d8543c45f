#include "dense_nt.hpp"

namespace rsvd {
DENSE_NT(DK_BF16, true)
}  // namespace rsvd
