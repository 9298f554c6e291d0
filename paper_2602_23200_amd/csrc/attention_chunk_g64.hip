// The kernels of attention_chunk.hip for groups of 64.
#define INNERQ_CHUNK_G 64
#include "attention_chunk.hip"
