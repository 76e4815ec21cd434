// Norms and joins of rows of fp32.
#include "join.hpp"

namespace rsh {
RSH_JOIN_OF(F32)
}
