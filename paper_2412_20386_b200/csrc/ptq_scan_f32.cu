// The scan of binary32 activations.
#define PTQ_SCAN_TYPE float
#include "ptq_scan_launch.cuh"
