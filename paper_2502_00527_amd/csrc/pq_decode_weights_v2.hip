// The kernels of pq_decode_weights.hip for 2-bit quantized values.
#define PQ_WEIGHTS_VB 2
#define PQ_WEIGHTS_LAUNCH launch_weights_v2
#include "pq_decode_weights.hip"
