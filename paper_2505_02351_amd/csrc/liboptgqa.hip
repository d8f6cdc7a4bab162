// The whole library as one source, for builds that take a single file; build.py compiles the parts side by side.
#include "optgqa.hip"
#include "operators.hip"
#include "pages.hip"
