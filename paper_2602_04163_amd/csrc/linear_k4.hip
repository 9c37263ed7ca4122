// The product on stored planes (linear.h), 4 planes per weight.
#include "linear.h"

namespace bpdq {
template int linear_run<4>(const LinearArgs&, int, hipStream_t);
}
