// New rows into the cache (norm of each head, rotation by position, 8-bit codes) and rows out of it again.
#include "cache.h"
#include "wave_util.h"

namespace obc {
namespace {

constexpr int kThreads = 256;
constexpr int kGroups = kThreads / 16;       // 16 lanes hold one row

// kN consecutive channels of a row, in fp32.
template <int kN, bool kBf16>
struct Raw { uint32_t w[kBf16 ? kN / 2 : kN]; };
template <int kN, bool kBf16>
__device__ __forceinline__ void widen(const Raw<kN, kBf16> &raw, float (&x)[kN]) {
    if constexpr (kBf16) {
        const uint32_t *w = raw.w;
#pragma unroll
        for (int i = 0; i < kN / 2; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kN; ++i) x[i] = __uint_as_float(raw.w[i]);
    }
}
template <int kN, bool kBf16, bool kPast>
__device__ __forceinline__ void store_row(char *p, const float (&x)[kN]) {
    if constexpr (kBf16) {
        uint32_t w[kN / 2];
#pragma unroll
        for (int i = 0; i < kN / 2; ++i) w[i] = bf16_pair_of(x[2 * i], x[2 * i + 1]);
        store_bytes<2 * kN, kPast>(p, w);
    } else {
        store_bytes<4 * kN, kPast>(p, x);
    }
}

// Row `j` of head h of sequence b (a row that the cache has no room for is dropped): this lane's kN channels from lo on.  A block of 32
// channels lies in 4 lanes (8 of half as many), which find its power of two together.
template <int kN, bool kBf16, bool kCodes, bool kPast>
__device__ __forceinline__ void put_row(const CacheView &c, char *pages, uint8_t *scales, int b, int h, long long at, int lo, const float (&x)[kN]) {
    constexpr int kD = 16 * kN, kSize = kBf16 ? 2 : 4;
    if (at < 0 || at >= c.capacity) return;
    const int j = (int)at, page = c.table ? c.table[(size_t)b * c.pages_per_seq + (j >> c.shift)] : b;
    if (page < 0 || page >= c.num_pages) return;
    const size_t row = row_in_pool(c, page, h, j);
    if constexpr (!kCodes) {
        store_row<kN, kBf16, kPast>(pages + row * (kD * kSize) + lo * kSize, x);
    } else {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < kN; ++i) top = fmaxf(top, finite_abs(x[i]));
        top = fmaxf(top, dpp_pair<0xB1>(top));
        top = fmaxf(top, dpp_pair<0x4E>(top));
        if constexpr (kN == 4) top = fmaxf(top, dpp_pair<0x141>(top));
        const uint32_t byte = scale_byte(top);
        const float inv = scale_inverse(byte);
        uint32_t w[kN / 4];
#pragma unroll
        for (int i = 0; i < kN; i += 4) w[i / 4] = e4m3_codes(x[i] * inv, x[i + 1] * inv, x[i + 2] * inv, x[i + 3] * inv);
        store_bytes<kN, kPast>(pages + row * kD + lo, w);
        if (lo % kScaleBlock == 0) scales[row * (kD / kScaleBlock) + lo / kScaleBlock] = (uint8_t)byte;
    }
}

// Rows that are stored as they are: 16 of a head per workgroup, so that neighbours in a page (and their scale bytes) are written together; K
// and V in one launch.
template <int kD, int kDtype, bool kCodes>
__global__ __launch_bounds__(kThreads) void store_rows(AppendArgs a) {
    constexpr int kN = kD / 16, kSize = kDtype == OBC_BF16 ? 2 : 4;
    const int t = blockIdx.x * kGroups + threadIdx.x / 16, lo = threadIdx.x % 16 * kN;
    const int b = blockIdx.y / a.cache.Hkv, g = blockIdx.y % a.cache.Hkv;
    const int n = a.fresh.len ? min(max(device_len(a.fresh, b, g, a.cache.Hkv), 0), a.T) : a.T;
    if (t >= n) return;
    const RowsView &from = blockIdx.z == 0 ? a.k : a.v;
    Raw<kN, kDtype == OBC_BF16> raw;
    load_bytes<kN * kSize>(raw.w, from.base + b * from.batch + t * from.token + g * from.head + lo * kSize);
    float x[kN];
    widen<kN, kDtype == OBC_BF16>(raw, x);
    put_row<kN, kDtype == OBC_BF16, kCodes, false>(a.cache, blockIdx.z == 0 ? a.cache.k : a.cache.v, blockIdx.z == 0 ? a.cache.k_scale : a.cache.v_scale,
                                                   b, g, (long long)device_len(a.lens, b, g, a.cache.Hkv) - n + t, lo, x);
}

// One workgroup per new token (and per 16 * gridDim.y of its heads): a row of d channels lies in 16 lanes, so the sum of its
// squares is four lane exchanges, and a lane keeps its channels' norm weights, cosines and sines for all heads of the token.
// The angle pos * f is reduced to a part of one turn in 64 bits: in fp32 the product alone would be off by 2^-24 of the angle,
// 0.06 rad at a million tokens.
//
// Bound by HBM, with the vector work beside it: 8192 tokens of 32/8 heads in bf16 (201 MB) 48 us; without norm and rotation 38.5, a copy of as many
// bytes 39.0.  A single token: 3.4 us, the launch and its trips to memory.
template <int kD, int kDtype, bool kCodes, bool kPast>
__global__ __launch_bounds__(kThreads) void append_rows(AppendArgs a) {
    constexpr int kN = kD / 16;
    constexpr bool kBf16 = kDtype == OBC_BF16;
    constexpr int kSize = kBf16 ? 2 : 4;
    __shared__ float2 turn[kD / 2];
    const int b = blockIdx.x / a.T, t = blockIdx.x % a.T;
    const int group = threadIdx.x / 16, c = threadIdx.x % 16, lo = kN * c;
    const int Hkv = a.cache.Hkv, rows = a.Hq + 2 * Hkv;
    const int first = blockIdx.y * kGroups + group, step = kGroups * gridDim.y;
    using R = Raw<kN, kBf16>;
    const char *q_in = a.q.base + b * a.q.batch + t * a.q.token, *k_in = a.k.base + b * a.k.batch + t * a.k.token;
    const char *v_in = a.v.base + b * a.v.batch + t * a.v.token;
    const auto fetch = [&](int r) {                        // (one kind per branch: its strides stay scalar)
        R raw;
        if (r < a.Hq) load_bytes<kN * kSize>(raw.w, q_in + r * a.q.head + lo * kSize);
        else if (r < a.Hq + Hkv) load_bytes<kN * kSize>(raw.w, k_in + (r - a.Hq) * a.k.head + lo * kSize);
        else load_bytes<kN * kSize>(raw.w, v_in + (r - a.Hq - Hkv) * a.v.head + lo * kSize);
        return raw;
    };
    R ahead = {};                                          // (us, without and with: 8192 tokens in bf16 48.9 and 50.1, 2048 in 8 bits 14.2 and 12.7)
    if (kCodes && first < rows) ahead = fetch(first);
    if (a.pairs) {
        for (int i = threadIdx.x; i < a.pairs; i += kThreads) {
            double turns = (double)a.positions[(size_t)b * a.T + t] * (double)a.inv_freq[i] * 0.15915494309189533577;
            turns -= rint(turns);
            float sn, cs;
            if constexpr (kBf16) {           // the instructions take turns; off by 1.3e-7 at most, here and for bf16 far below the result's rounding
                sn = __builtin_amdgcn_sinf((float)turns);
                cs = __builtin_amdgcn_cosf((float)turns);
            } else {
                sincospif(2.f * (float)turns, &sn, &cs);
            }
            turn[i] = make_float2(cs * a.rot_scale, sn * a.rot_scale);
        }
        __syncthreads();
    }
    // channels lo .. lo + kN - 1: their angles, and for pairs (i, i + pairs) the lane that holds the other ones
    const bool turned = lo < 2 * a.pairs, second = lo >= a.pairs;
    const int partner = (threadIdx.x & 48) + (second ? c - a.pairs / kN : c + a.pairs / kN);
    float cs[kN], sn[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const float2 x = turned ? turn[a.interleaved ? (lo + i) / 2 : second ? lo + i - a.pairs : lo + i] : make_float2(1.f, 0.f);
        cs[i] = x.x;
        sn[i] = (a.interleaved ? i % 2 == 0 : !second) ? -x.y : x.y;
    }
    const int exchange = !a.pairs ? 0 : a.interleaved ? 1 : 2 * a.pairs == kD ? 2 : 3;

    // Row r of the token: norm and rotation.
    const auto form = [&](const R &raw, const void *norm, float (&x)[kN]) {
        widen<kN, kBf16>(raw, x);
        if (norm) {
            R weights;
            float w[kN], sum = 0.f;
            load_bytes<kN * kSize>(weights.w, (const char *)norm + lo * kSize);
            widen<kN, kBf16>(weights, w);
#pragma unroll
            for (int i = 0; i < kN; ++i) sum = fmaf(x[i], x[i], sum);
            const float inv = rsqrtf(row16_reduce<SumOp>(sum) * (1.f / kD) + a.eps);
#pragma unroll
            for (int i = 0; i < kN; ++i) x[i] = x[i] * inv * w[i];
        }
        if (exchange == 0) return;
        float y[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i) y[i] = exchange == 1 ? x[i ^ 1] : exchange == 2 ? dpp_pair<0x128>(x[i]) : __shfl(x[i], partner);
        // (a selection, no angle of 0: 0 times another lane's infinity is no 0)
#pragma unroll
        for (int i = 0; i < kN; ++i) x[i] = turned ? fmaf(x[i], cs[i], y[i] * sn[i]) : x[i];
    };
    const auto store = [&](int h, int n, char *pages, uint8_t *scales, const float (&x)[kN]) {
        put_row<kN, kBf16, kCodes, kPast>(a.cache, pages, scales, b, h, (long long)device_len(a.lens, b, h, Hkv) - n + t, lo, x);
    };
    for (int r = first; r < rows; r += step) {
        const int g = r < a.Hq ? 0 : r < a.Hq + Hkv ? r - a.Hq : r - a.Hq - Hkv;
        const int n = a.fresh.len ? min(max(device_len(a.fresh, b, g, Hkv), 0), a.T) : a.T;
        float x[kN];
        R raw;
        if constexpr (kCodes) {
            raw = ahead;
            if (r + step < rows) ahead = fetch(r + step);
        }
        if (r < a.Hq) {
            if (t < n) {
                if constexpr (!kCodes) load_bytes<kN * kSize>(raw.w, q_in + r * a.q.head + lo * kSize);
                form(raw, a.q_norm, x);
            } else {
#pragma unroll
                for (int i = 0; i < kN; ++i) x[i] = 0.f;
            }
            store_row<kN, kBf16, kPast>(a.q_out + (((size_t)b * a.Hq + r) * a.T + t) * (kD * kSize) + lo * kSize, x);
        } else if (t >= n) {
            continue;
        } else if (r < a.Hq + Hkv) {
            if constexpr (!kCodes) load_bytes<kN * kSize>(raw.w, k_in + g * a.k.head + lo * kSize);
            form(raw, a.k_norm, x);
            store(g, n, a.cache.k, a.cache.k_scale, x);
        } else {
            if constexpr (!kCodes) load_bytes<kN * kSize>(raw.w, v_in + g * a.v.head + lo * kSize);
            widen<kN, kBf16>(raw, x);
            store(g, n, a.cache.v, a.cache.v_scale, x);
        }
    }
}

// Rows of the cache as bf16 or fp32, kPer channels per thread; a head's rows per grid column, K and V in one launch.  (With threads numbered
// through, the 64-bit divisions that find a row's head cost more than its way: 4 x 8 heads x 2048 bf16 rows 14.4 us, now 12.2, a copy of as many
// bytes 13.7; x 8192 60.9 and 54.2.)  Stored past the caches at every size: from 4 x 8 heads x 2048 bf16 rows on that takes 7 to 10 % off a read (54.1 and
// 58.2 us x 8192; of 8-bit rows 40.0 and 47.4) and puts 0 to 3 % on a read with obc_score of 32 rows behind it (133.4 and 129.0; 121.8 and 118.5; x 2048 the same).
template <int kD, int kDtype, bool kCodes, int kPer>
__global__ __launch_bounds__(kThreads) void read_rows(ReadArgs a) {
    constexpr int kPieces = kD / kPer, kSize = kDtype == OBC_BF16 ? 2 : 4;
    const unsigned at = blockIdx.x * kThreads + threadIdx.x;
    const int i = (int)(at / kPieces), lo = (int)(at % kPieces) * kPer;
    if (i >= a.n) return;
    const int b = blockIdx.y / a.cache.Hkv, g = blockIdx.y % a.cache.Hkv;
    const size_t out_row = (size_t)blockIdx.y * a.n + i;
    int j = a.keep ? a.keep[out_row] : i;
    char *to = (blockIdx.z == 0 ? a.k_out : a.v_out) + out_row * (kD * kSize) + lo * kSize;
    const bool none = j < 0;
    j = min(max(j, 0), a.cache.capacity - 1);
    const size_t row = row_in_pool(a.cache, page_of(a.cache, b, j), g, j);
    const char *pages = blockIdx.z == 0 ? a.cache.k : a.cache.v;
    if constexpr (kCodes) {
        const uint8_t *scales = blockIdx.z == 0 ? a.cache.k_scale : a.cache.v_scale;
        uint32_t w[kPer / 4] = {};
        if (!none) load_bytes<kPer>(w, pages + row * kD + lo);
        const float s = none ? 0.f : scale_value(scales[row * (kD / kScaleBlock) + lo / kScaleBlock]);
        float z[kPer];
#pragma unroll
        for (int q = 0; q < kPer / 4; ++q) {
            float y[4];
            e4m3_values(w[q], s, y);
#pragma unroll
            for (int e = 0; e < 4; ++e) z[4 * q + e] = y[e];
        }
        store_row<kPer, kDtype == OBC_BF16, true>(to, z);
    } else {
        uint32_t x[kPer * kSize / 4] = {};
        if (!none) load_bytes<kPer * kSize>(x, pages + row * (kD * kSize) + lo * kSize);
        store_bytes<kPer * kSize, true>(to, x);
    }
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, hipStream_t stream) {
    const int rows = a.Hq + 2 * a.cache.Hkv;
    const unsigned tokens = (unsigned)(a.B * a.T);
    const unsigned groups = (rows + kGroups - 1) / kGroups;
    const unsigned y = tokens < 1024 ? groups : 1;       // few tokens: every row a group of its own
    if (!a.Hq && !a.pairs && !a.k_norm) {
        const dim3 grid((a.T + kGroups - 1) / kGroups, a.B * a.cache.Hkv, 2);
        return with_types(a.d, a.dtype, a.cache_dtype, [&](auto dim, auto type, auto codes) {
            store_rows<dim.value, type.value, codes.value><<<grid, kThreads, 0, stream>>>(a);
            return hipGetLastError();
        });
    }
    // bf16 rows are stored past the caches from 8 MiB of them on (us, kept and past, 32/8 heads of 128 channels; 2048, 4096, 8192, 16384 tokens: inputs from
    // HBM 19.2 and 18.6, 29.9 and 28.7, 50.5 and 48.5, 94.3 and 90.9; from the caches 13.8 and 12.3, 21.5 and 20.5, 35.9 and 35.7, 93.3 and 67.3; with obc_attend behind it
    // alike to 0.6 of 65 to 560).  fp32 rows, and rows that are stored as they are, not: from HBM the former gain 0.5 of 27.8 (2048 tokens) and lose 4.2 of 20.6
    // from the caches; of the latter 2048 x 32 heads into 8 bits take 22.1 and 26.1 with the read behind them, 16384 x 8 in fp32 41.0 and 55.7.
    const bool past = a.dtype == OBC_BF16 && (size_t)tokens * rows * a.d * 2 > ((size_t)8 << 20);
    return with_types(a.d, a.dtype, a.cache_dtype, [&](auto dim, auto type, auto codes) {
        constexpr bool kMay = type.value == OBC_BF16;
        if (kMay && past) append_rows<dim.value, type.value, codes.value, kMay><<<dim3(tokens, y), kThreads, 0, stream>>>(a);
        else append_rows<dim.value, type.value, codes.value, false><<<dim3(tokens, y), kThreads, 0, stream>>>(a);
        return hipGetLastError();
    });
}

hipError_t launch_cache_read(const ReadArgs &a, hipStream_t stream) {
    // 16 codes per thread where there are rows enough (us, 8 and 16: 4 x 8 heads x 2048 rows 11.2 and 12.6, x 8192 52.4 and 43.3).  Not into fp32, where
    // a store then is a quarter of a thread's 64 bytes and those past the caches are not put together again (8 heads x 16384 rows 32.5 and 95.4).
    const int per = a.cache_dtype == OBC_E4M3 && a.dtype == OBC_BF16 && (size_t)a.B * a.cache.Hkv * a.n >= (1u << 17) ? 16 : 8;
    const unsigned pieces = (unsigned)a.n * (a.d / per);
    const dim3 grid((pieces + kThreads - 1) / kThreads, a.B * a.cache.Hkv, 2);
    return with_types(a.d, a.dtype, a.cache_dtype, [&](auto dim, auto type, auto codes) {
        constexpr int kMost = codes.value && type.value == OBC_BF16 ? 16 : 8;
        if (per == kMost) read_rows<dim.value, type.value, codes.value, kMost><<<grid, kThreads, 0, stream>>>(a);
        else read_rows<dim.value, type.value, codes.value, 8><<<grid, kThreads, 0, stream>>>(a);
        return hipGetLastError();
    });
}

}  // namespace obc
