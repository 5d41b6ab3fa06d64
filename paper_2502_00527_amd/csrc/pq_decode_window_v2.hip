// The sliding-window kernels of pq_decode_window.hip for 2-bit quantized values.
#define PQ_WINDOW_VB 2
#define PQ_WINDOW_LAUNCH launch_window_v2
#include "pq_decode_window.hip"
