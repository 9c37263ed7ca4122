// The gated product on stored planes (linear.h), 2 planes per weight.
#include "linear.h"

namespace bpdq {
template int linear_run<2, true>(const LinearArgs&, int, hipStream_t);
}
