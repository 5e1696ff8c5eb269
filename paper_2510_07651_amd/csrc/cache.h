// The cache that kept and new rows live in, as the kernels see it, and its 8-bit number format.
// Internal to the library.
#pragma once

#include <type_traits>

#include "internal.h"

namespace obc {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16_pair __attribute__((ext_vector_type(2)));
typedef float f32_pair __attribute__((ext_vector_type(2)));

// Pages of `slots` = 2^shift rows per KV head; without a table sequence b is page b, which holds all of its rows.
struct CacheView {
    char *k, *v;
    uint8_t *k_scale, *v_scale;
    const int32_t *table;
    int num_pages, pages_per_seq, page_size, shift, Hkv, capacity;   // shift: 31 without a table
};

// Device lengths: one per sequence, or one per (sequence, KV head).
struct DeviceLens {
    const int32_t *len;
    int per_head;
};
__device__ __forceinline__ int device_len(const DeviceLens &l, int b, int g, int Hkv) {
    return l.len[l.per_head ? b * Hkv + g : b];
}

// Row index inside the pool, in rows, of row `j` of KV head g: page * Hkv * slots + g * slots + slot.  64 bits: a pool may have more
// than 2^31 elements.  Page numbers are device data that nobody has checked: outside the pool they are brought inside.
__device__ __forceinline__ int page_of(const CacheView &c, int b, int j) {
    const int p = c.table ? c.table[(size_t)b * c.pages_per_seq + (j >> c.shift)] : b;
    return min(max(p, 0), c.num_pages - 1);
}
__device__ __forceinline__ size_t row_in_pool(const CacheView &c, int page, int g, int j) {
    return ((size_t)page * c.Hkv + g) * c.page_size + (j & ((1u << c.shift) - 1));
}

// ---- e4m3 with one power of two per 32 channels ----------------------------------------------------------------------------
// The stored byte is e + 127 with e the least integer for which absmax <= 448 * 2^e (absmax of the block's finite values), at
// least -117, so that every value a code stands for is a normal fp32 (and bf16) number: 2^-9 * 2^-117 = 2^-126.  448 = 1.75 * 2^8.
// Dividing by 2^e is exact and multiplying back is too, in bf16 as well (four significant bits): the only rounding is the one
// to the code, and rows that are read back and stored again keep their values.  (Only values that round to 2^128 have no place in fp32: they
// are read back as infinity.)
constexpr int kScaleBlock = 32;
constexpr uint32_t kLeastScale = 10;
__device__ __forceinline__ uint32_t scale_byte(float absmax) {
    const uint32_t u = __float_as_uint(absmax);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(e, (int)kLeastScale);
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a < __builtin_inff() ? a : 0.f;
}
__device__ __forceinline__ float finite_or_nan(float x) { return fabsf(x) < __builtin_inff() ? x : __builtin_nanf(""); }
// Four values (already divided by their power of two) to codes, rounded to nearest even.  An infinity or NaN becomes NaN.
__device__ __forceinline__ uint32_t e4m3_codes(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(finite_or_nan(a), finite_or_nan(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(finite_or_nan(c), finite_or_nan(d), w, true);
}
__device__ __forceinline__ void e4m3_values(uint32_t codes, float scale, float (&x)[4]) {
    const f32_pair lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    x[0] = lo[0] * scale; x[1] = lo[1] * scale; x[2] = hi[0] * scale; x[3] = hi[1] * scale;
}
// Four codes to four bf16 values, exactly.
__device__ __forceinline__ u32x2 e4m3_bf16(uint32_t codes, float scale) {
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes, scale, false);
    const auto hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes, scale, true);
    return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}
__device__ __forceinline__ uint32_t bf16_pair_of(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32_pair){lo, hi}, bf16_pair));   // to nearest even
}

// kBytes (4, 8 or a multiple of 16) between memory, as aligned as they are many, and a local array of any type.
template <int kBytes>
__device__ __forceinline__ void load_bytes(void *to, const void *p) {
    if constexpr (kBytes == 4) {
        const uint32_t x = *(const uint32_t *)p;
        __builtin_memcpy(to, &x, 4);
    } else if constexpr (kBytes == 8) {
        const u32x2 x = *(const u32x2 *)p;
        __builtin_memcpy(to, &x, 8);
    } else {
#pragma unroll
        for (int i = 0; i < kBytes / 16; ++i) {
            const u32x4 x = *((const u32x4 *)p + i);
            __builtin_memcpy((char *)to + 16 * i, &x, 16);
        }
    }
}
// `kPast`: past the caches.
template <int kBytes, bool kPast>
__device__ __forceinline__ void store_bytes(void *p, const void *from) {
    const auto put = [](auto *to, const auto &x) {
        if constexpr (kPast) __builtin_nontemporal_store(x, to);
        else *to = x;
    };
    if constexpr (kBytes == 4) {
        uint32_t x;
        __builtin_memcpy(&x, from, 4);
        put((uint32_t *)p, x);
    } else if constexpr (kBytes == 8) {
        u32x2 x;
        __builtin_memcpy(&x, from, 8);
        put((u32x2 *)p, x);
    } else {
#pragma unroll
        for (int i = 0; i < kBytes / 16; ++i) {
            u32x4 x;
            __builtin_memcpy(&x, (const char *)from + 16 * i, 16);
            put((u32x4 *)p + i, x);
        }
    }
}

// ---- what the calls hand to the launchers ----------------------------------------------------------------------------------
struct RowsView {            // rows of d contiguous elements at base + b * batch + t * token + h * head (bytes)
    const char *base;
    int64_t batch, token, head;
};
struct AppendArgs {
    RowsView q, k, v;        // q.base may be null
    CacheView cache;
    char *q_out;             // [B,Hq,T,d]
    DeviceLens lens, fresh;  // fresh.len null: T new rows everywhere
    const int32_t *positions;
    const float *inv_freq;
    int pairs;               // 0: no rotation
    float rot_scale;
    int interleaved;
    const void *q_norm, *k_norm;
    float eps;
    int B, T, Hq, d, dtype, cache_dtype;
};
struct ReadArgs {
    CacheView cache;
    const int32_t *keep;     // [B,Hkv,n] or null: rows 0 .. n-1
    char *k_out, *v_out;
    int B, n, d, dtype, cache_dtype;
};
struct AttendArgs {
    const char *q;           // [B,Hq,T,d]
    CacheView cache;
    char *out;               // [B,T,Hq,d]
    DeviceLens lens;
    const int32_t *fresh;    // [B] or null
    int B, T, Hq, Hkv, G, d, dtype, cache_dtype, causal;
    float scale_log2;        // scale * log2(e)
};
// How a call is cut up: rows (query head, new token) of a KV head in tiles, tokens in `splits` shares.  Offsets into the workspace.
enum { kAttendFp32 = 0, kAttendChunk = 1, kAttendToken = 2 };
struct AttendPlan {
    int form;                // kernel
    int tiles, tile_rows, splits;
    int step, min_share;     // a share: a multiple of `step` tokens, at least `min_share`
    size_t part_ml, part_o, total;
};

// Calls `f` with a kernel's compile-time choices.
template <typename F>
hipError_t with_types(int d, int dtype, int cache_dtype, F &&f) {
    const bool codes = cache_dtype == OBC_E4M3;
    using std::integral_constant;
    const auto by_codes = [&](auto dim, auto type) {
        return codes ? f(dim, type, std::true_type()) : f(dim, type, std::false_type());
    };
    const auto by_type = [&](auto dim) {
        return dtype == OBC_BF16 ? by_codes(dim, integral_constant<int, OBC_BF16>()) : by_codes(dim, integral_constant<int, OBC_F32>());
    };
    return d == 128 ? by_type(integral_constant<int, 128>()) : by_type(integral_constant<int, 64>());
}

hipError_t launch_append(const AppendArgs &a, hipStream_t stream);
hipError_t launch_cache_read(const ReadArgs &a, hipStream_t stream);
void plan_attend(int B, int T, int Hq, int Hkv, int d, int capacity, int dtype, int cache_dtype, AttendPlan *p);
hipError_t launch_attend(const AttendArgs &a, const AttendPlan &p, char *workspace, hipStream_t stream);

}  // namespace obc
