// What the attention kernels share: tiles of rows, shares of the sequence, partial results.  Internal to the library.
//
// The rows (new token t, query head h of a KV head) of one KV head read the same keys and values, so they are taken together,
// token by token: row r is token r / G of query head g G + r % G, and a tile of consecutive rows sees nearly the same tokens.
#pragma once

#include "cache.h"

namespace obc {

constexpr int kAttendChunkRows = 128;  // rows per workgroup of attend_chunk
// A row's weights are 2^(logit - reference), with logits in log2, and at most 1, so that sums of N values below 2^127 / N have a place in fp32.  The
// reference is set kLazy above the largest logit so far, and moved, with the sums rescaled, when a logit passes it.  In fp32 it is set closer: the largest
// weights' exponents, logit - reference, are rounded to half an ulp of it, 2^-23 at 2 and 2^-21 at 8, which only a weight that becomes bf16 can bear.
constexpr float kLazy = 8.f, kLazyFp32 = 2.f;
constexpr float kNone = -3.0e38f;      // running maximum of a row that has seen nothing: finite, so that differences stay numbers

struct Tile {            // rows r0 .. r0 + size - 1 of KV head g of sequence b
    int b, g, r0, len, n, seen;      // len: rows of the KV head, also those for which the cache had no room; n: new tokens; seen: the most any row sees
    // Tokens that the rows of new token t see, if the cache had room for all: the token's own row is row len - n + t.
    __device__ __forceinline__ int sees(int t, int causal) const {
        if (t >= n) return 0;
        return causal ? max(len - n + t + 1, 0) : len;
    }
};
__device__ __forceinline__ Tile tile_of(const AttendArgs &a, int bg, int r0, int size) {
    Tile x;
    x.b = bg / a.Hkv;
    x.g = bg % a.Hkv;
    x.r0 = r0;
    x.len = min(max(device_len(a.lens, x.b, x.g, a.Hkv), 0), a.cache.capacity + a.T);    // (from there on every new token sees the whole cache)
    x.n = a.fresh ? min(max(a.fresh[x.b], 0), a.T) : a.T;
    const int first = r0 / a.G, last = min((r0 + size - 1) / a.G, x.n - 1);
    x.seen = first <= last ? min(x.sees(last, a.causal), a.cache.capacity) : 0;
    return x;
}
// Tokens per share of a tile: the same in the kernels that leave partial sums and in the one that joins them.  A sequence that is short
// for its cache has fewer shares than the plan.
__device__ __forceinline__ int share_of(int seen, const AttendPlan &p) {
    const int even = (seen + p.splits - 1) / p.splits;
    return max((even + p.step - 1) / p.step * p.step, p.min_share);
}

template <int kDtype>
__device__ __forceinline__ void store4(void *p, const float (&x)[4]) {
    if constexpr (kDtype == OBC_BF16) {
        const uint32_t w[2] = {bf16_pair_of(x[0], x[1]), bf16_pair_of(x[2], x[3])};
        store_bytes<8, false>(p, w);
    } else {
        store_bytes<16, false>(p, x);
    }
}

hipError_t launch_attend_token(const AttendArgs &a, const AttendPlan &p, float2 *part_ml, float *part_o, hipStream_t stream);
hipError_t launch_attend_chunk(const AttendArgs &a, const AttendPlan &p, float2 *part_ml, float *part_o, hipStream_t stream);

}  // namespace obc
