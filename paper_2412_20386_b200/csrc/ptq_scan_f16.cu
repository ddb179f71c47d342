// The scan of binary16 activations.
#define PTQ_SCAN_TYPE __half
#include "ptq_scan_launch.cuh"
