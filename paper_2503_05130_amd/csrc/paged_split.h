// How paged attention splits a request's keys into parts, one workgroup each per
// key-value head and 16 of its query heads.  Host and device code share it (the
// workspace is sized by the same rule).
#pragma once

#include <hip/hip_runtime.h>

namespace iefwd {

// Query heads of one key-value head are worked on in tiles of 16, the width
// of one MFMA operand.
inline __host__ __device__ int paged_tiles(int n_heads, int n_kv_heads) { return (n_heads / n_kv_heads + 15) / 16; }

// With `rows` = batch x key-value heads x tiles, in classes of a factor of two, a
// request is cut into up to 256 / rows parts (at most 64), so that one request alone gives
// every CU a workgroup.  A part has a power of two of keys, from 256 to 1024 and more only past
// 128 parts: one long request among short ones must not be left to a few workgroups.
// Measured with parts of 256, 512 and 1024 keys (us; 32 query and 8 key-value heads of 128 unless
// stated):
//   1 x 4000 keys        10.6 11.0 13.4      16 x 2000               27.7 26.9 26.4
//   1 x 32001            29.3 27.5 26.1      64 x 4000 - 8192         275  260  250
//   96 x 5 - 12000, 16 / 4 heads of 64, e4m3 26.6 23.5 22.2
// A request of up to 512 keys is never split: the launch that joins its parts would cost more
// (1 x 300: 8.2 in parts of 256, 5.7 in one).
// A workgroup has 8 waves.  From 4096 rows on, more than the chip holds several times over, it has 2: a long
// request's rows keep it busy all the same, and a short one's leave fewer waves idle (us with 8 / 4 / 2 waves:
// 1024 x 20 - 60 keys, 8 heads of 64, 57 / 40 / 26; 1024 x 200 - 400, 32 / 8 heads of 128, 203 / 202 / 202; but
// 256 x 800 - 1600 211 / 215 / 223; one request of 1000 8.3 / 8.5 with 8 / 4).
constexpr int kPagedWholeLog2 = 9, kPagedMinLog2 = 8, kPagedMaxLog2 = 10;

struct PagedSplit {
    int log2_parts;   // up to this many parts (log2)
    int waves;        // of a workgroup
};

inline __host__ __device__ int log2_up(int n) { return n <= 1 ? 0 : 32 - __builtin_clz((unsigned)(n - 1)); }

inline __host__ __device__ PagedSplit paged_split(int batch, int n_heads, int n_kv_heads) {
    const long rows = (long)batch * n_kv_heads * paged_tiles(n_heads, n_kv_heads);
    const int spare = rows >= 256 ? 0 : 8 - log2_up((int)rows);
    return {spare < 6 ? spare : 6, rows >= 4096 ? 2 : 8};
}

// log2 of the keys in each part of a request of n_keys >= 0; from 513 keys on it never falls as n_keys grows
inline __host__ __device__ int paged_part_log2(int n_keys, PagedSplit s) {
    if (n_keys <= 1 << kPagedWholeLog2) return kPagedWholeLog2;
    const int even = log2_up((n_keys + (1 << s.log2_parts) - 1) >> s.log2_parts);
    const int most = log2_up((n_keys + 127) >> 7);      // for 128 parts
    const int part = even < kPagedMinLog2 ? kPagedMinLog2 : even > kPagedMaxLog2 ? kPagedMaxLog2 : even;
    return part < most ? most : part;
}

inline __host__ __device__ int paged_parts(int n_keys, PagedSplit s) {
    const int log2 = paged_part_log2(n_keys, s);
    return n_keys < 1 ? 1 : (n_keys + (1 << log2) - 1) >> log2;
}

// The most parts of any request of at most max_keys.  The count falls where the part
// doubles, so the longest request need not have the most.
inline int paged_most_parts(int max_keys, PagedSplit s) {
    int most = 1;
    for (int n = max_keys; n > 1 << kPagedWholeLog2;) {
        const int log2 = paged_part_log2(n, s), parts = paged_parts(n, s);
        if (parts > most) most = parts;
        int lo = 1 << kPagedWholeLog2, hi = n - 1;       // the longest with a smaller part
        while (lo < hi) {
            const int mid = lo + (hi - lo + 1) / 2;
            if (paged_part_log2(mid, s) < log2) lo = mid;
            else hi = mid - 1;
        }
        n = lo;
    }
    return most;
}

}  // namespace iefwd
