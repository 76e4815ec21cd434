// Norms and joins of rows of bfloat16.
#include "join.hpp"

namespace rsh {
RSH_JOIN_OF(BF16)
}
