// The classes that a draw keeps of every row: the kernels of sample.cu as far as
// the cut.
#define BITLOGIC_SUPPORT_UNIT
#include "sample.cu"
