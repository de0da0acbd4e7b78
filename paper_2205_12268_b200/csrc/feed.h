// What the thread that feeds a ring in shared memory may wait for (plain C++, no CUDA: a test compiles it by itself).
#pragma once

#ifdef __CUDACC__
#define WCC_ANYWHERE __host__ __device__ __forceinline__
#else
#define WCC_ANYWHERE inline
#endif

namespace wcc {

// The chunk whose release the feeder waits for once a tile's chunks first .. sent-1 are on their way, before it takes its next ticket: the tile's first one, so
// that a ticket is taken early enough to bring the next tile in on time, and no tile waits behind another while a CTA has nothing to do.  -1: none.  With more
// chunks than stages, sending the last of them has waited for the first already, and must not be waited for again: a wait by parity is over while one
// completion of the stage's barrier has happened since, and with two (chunk first + stages let go as well) it would be for a chunk that is not sent yet.
WCC_ANYWHERE int awaited_chunk(int first, int sent, int stages) { return first + stages < sent ? -1 : first; }

}  // namespace wcc
