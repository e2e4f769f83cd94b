// Arguments and launchers of the operators beside the index: heads.hip, packed.hip, tree.hip.
#pragma once

#include "common.hpp"

namespace dynakv {

// Calls that move more than the memory-side cache holds leave nothing in it that a later one could find: they load and store past the caches
// (STREAM), so that what is there of others stays.  Smaller calls do not, for the kernel that reads their rows next.
constexpr long long kCacheBytes = 256ll << 20;
template <bool STREAM, class T>
__device__ __forceinline__ T get(const T* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool STREAM, class T>
__device__ __forceinline__ void put(T* p, T x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, p);
  else *p = x;
}

struct HeadsArgs {
  dynakv_heads_t c;
  const void *q, *k, *v, *wq, *wk;
  const float* inv_freq;
  const int* positions;
  void *Q, *K, *V;
  int per;   // rows of a token that each row of 16 lanes works on
};
hipError_t launch_norm_rope(const HeadsArgs& a, hipStream_t st);

// ---- packed cache ---------------------------------------------------------------------------------------------
constexpr int kBlock = 32;                          // values that share a scale
constexpr int kRowScales = kHeadDim / kBlock;       // scale bytes of a row
__host__ __device__ inline int code_bytes(int bits) { return kHeadDim * bits / 8; }
// Scale byte -> 2^(s - 127); 255: NaN.
__device__ __forceinline__ float scale_value(uint32_t s) {
  return __uint_as_float(s == 255u ? 0x7FC00000u : s ? s << 23 : 0x00400000u);
}
hipError_t launch_packed_write(const dynakv_packed_t& c, const void* K, const void* V, int n, const int* start, const int* count,
                               hipStream_t st);
hipError_t launch_packed_read(const dynakv_packed_t& c, const int* positions, int n, void* K, void* V, hipStream_t st);

// ---- attention of drafted tokens --------------------------------------------------------------------------------
constexpr int kMaxNodes = 64;                       // one bit each in a node's word of the tree
struct TreeArgs {
  int U, T, G, dtype;
  float sc;                                         // softmax scale * log2(e)
  const void *Q, *K1, *V1;
  const unsigned long long* tree;                   // null: a chain
  void* out;
  float* lse;
  void* scratch;
  int most;                                         // what the cut is planned for: a unit's tokens at most, as far as the host knows (the capacity, the
                                                    // budget; a list of clusters of one token has four slots for each, of which one is used)
  // the entries: the gather list of an index ...
  const char* pages;                                // null: a packed cache
  size_t unit_pages;                                // bytes of a unit's page pool
  const int *plist, *n_list;
  int Lcap;
  // ... or rows of a packed cache
  dynakv_packed_t cache;
  const int* lengths;
  // set by launch_tree
  int RB, rows;                                     // blocks of rows of a unit, rows of each
  int pieces;                                       // most workgroups for each; U: every unit whole
  int least;                                        // entries for which another workgroup is worth it
  int* where;                                       // [U][2] first piece and pieces of a unit
  float* part;                                      // [pieces][T * G][kPartRow]
};
constexpr int kPartRow = kHeadDim + 4;              // accumulators, maximum, both sums of weights, padding to 16 bytes
size_t tree_scratch_bytes(int U, int T, int G);
hipError_t launch_tree(const TreeArgs& a, hipStream_t st);

}  // namespace dynakv
