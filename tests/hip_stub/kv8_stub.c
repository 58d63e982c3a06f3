/* The stand-in HIP runtime with what the calls of the paged 8-bit cache ask for beside it: the current device. */
#include "hip_stub.c"
static int device;
int hipGetDevice(int *d) { *d = device; return 0; }
