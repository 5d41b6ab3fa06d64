// The sliding-window kernels of pq_decode_window.hip for 4-bit quantized values.
#define PQ_WINDOW_VB 4
#define PQ_WINDOW_LAUNCH launch_window_v4
#include "pq_decode_window.hip"
