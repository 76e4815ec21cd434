// Norms and joins of rows of binary16.
#include "join.hpp"

namespace rsh {
RSH_JOIN_OF(F16)
}
