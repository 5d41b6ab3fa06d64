// Chunk attention over 2-bit values.
#define PQ_CHUNK_VB 2
#define PQ_CHUNK_LAUNCH launch_chunk_v2
#include "pq_chunk_attention.hip"
