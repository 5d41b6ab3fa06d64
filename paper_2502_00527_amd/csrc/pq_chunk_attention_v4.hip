// Chunk attention over 4-bit values.
#define PQ_CHUNK_VB 4
#define PQ_CHUNK_LAUNCH launch_chunk_v4
#include "pq_chunk_attention.hip"
