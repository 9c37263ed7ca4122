// The product on stored planes (linear.h), 2 planes per weight.
#include "linear.h"

namespace bpdq {
template int linear_run<2, false>(const LinearArgs&, int, hipStream_t);
}
