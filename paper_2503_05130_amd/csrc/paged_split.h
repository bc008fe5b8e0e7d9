// How paged attention splits a request's keys: into parts of one length, a
// multiple of 128 keys and at least 256, at most paged_max_parts() of them.
// Host and device code share it (the workspace is sized by the same rule).
#pragma once

#include <hip/hip_runtime.h>

namespace iefwd {

constexpr int kPagedMinPart = 256;

// Query heads of one key-value head are worked on in tiles of 16, the width
// of one MFMA operand.
inline __host__ __device__ int paged_tiles(int n_heads, int n_kv_heads) { return (n_heads / n_kv_heads + 15) / 16; }

// The most parts a request is cut into: together with the key-value heads about two
// workgroups a CU for a single request.  It depends on the head layout alone, never
// on the batch, so that a request's result does not depend on its neighbours.
inline __host__ __device__ int paged_max_parts(int n_heads, int n_kv_heads) {
    const int per_part = n_kv_heads * paged_tiles(n_heads, n_kv_heads);
    return per_part >= 16 ? 32 : 512 / per_part;
}

inline __host__ __device__ int paged_part_keys(int n_keys, int max_parts) {
    const int even = (n_keys + max_parts - 1) / max_parts;
    return even <= kPagedMinPart ? kPagedMinPart : (even + 127) / 128 * 128;
}

inline __host__ __device__ int paged_parts(int n_keys, int max_parts) {
    const int part = paged_part_keys(n_keys, max_parts);
    return (n_keys + part - 1) / part;
}

}  // namespace iefwd
