// Differences of whole numbers as the kernels take them, callable from the tests.
#include "common.hpp"

extern "C" void whole_differences(float* out, const int32_t* a, const int32_t* b, int less, int n)
{
    for (int i = 0; i < n; ++i) out[i] = optgqa::whole_difference(a[i], b[i], less);
}
