// attend_chunk_tree.cu -- attend_chunk.cu for drafted trees: a unit of its own, so that the two compile side by side and
// neither's code moves the other's.
#define CHUNK_TREE 1
#include "attend_chunk.cu"
