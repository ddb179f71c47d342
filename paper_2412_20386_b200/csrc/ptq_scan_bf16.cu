// The scan of bfloat16 activations.
#define PTQ_SCAN_TYPE __nv_bfloat16
#include "ptq_scan_launch.cuh"
