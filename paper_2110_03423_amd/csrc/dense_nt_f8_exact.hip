#include "dense_nt.hpp"

namespace rsvd {
DENSE_NT(DK_F8_EXACT, false)
}  // namespace rsvd
