#define PTQ_HEADS_DEFINE
#include "ptq_heads_launch.cuh"
template struct ptq_host::HeadsLaunch<__half>;
