// libsbw in one translation unit: the operators of sbw_step.h share the argument checks, the
// thread's last HIP error and the 16-byte vector types of the watermark's source.
#include "sbw_kernels.hip"
#include "sbw_logprobs.hip"
#include "sbw_head.hip"
