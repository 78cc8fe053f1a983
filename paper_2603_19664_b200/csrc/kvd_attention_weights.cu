// The launches of kvd_decode_attention_weights: the kernels of kvd_attention.cu with their WEIGH parameter set.  A unit of its
// own, so that the two sets of kernels compile side by side.
#define KVD_ATTENTION_WEIGHTS
#include "kvd_attention.cu"
