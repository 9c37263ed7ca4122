// The product on stored planes (linear.h), 1 plane per weight.
#include "linear.h"

namespace bpdq {
template int linear_run<1>(const LinearArgs&, int, hipStream_t);
}
