// The product on stored planes (linear.h), 3 planes per weight.
#include "linear.h"

namespace bpdq {
template int linear_run<3>(const LinearArgs&, int, hipStream_t);
}
