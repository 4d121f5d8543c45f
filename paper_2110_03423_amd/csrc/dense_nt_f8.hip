#include "dense_nt.hpp"

namespace rsvd {
DENSE_NT(DK_F8, false)
}  // namespace rsvd
