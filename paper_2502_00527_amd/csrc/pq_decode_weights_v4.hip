// The kernels of pq_decode_weights.hip for 4-bit quantized values.
#define PQ_WEIGHTS_VB 4
#define PQ_WEIGHTS_LAUNCH launch_weights_v4
#include "pq_decode_weights.hip"
