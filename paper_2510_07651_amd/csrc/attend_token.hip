// Attention of few rows per KV head (single tokens, up to 32 rows of query heads and new tokens) over the cache, bf16 queries.
//
// Every byte of the cache is used once, so nothing is staged: a wave loads keys and values of 32 tokens straight into the operand
// layout of the 16 x 16 x 32 matrix op.  S^T = K Q^T: lane l holds token l % 16 of a block of 16 and, per op, 8 channels.  The result
// has tokens 4 (l / 16) + r of both blocks in a lane's registers, for row l % 16.  O^T = V^T P^T takes its 8 tokens per lane in
// that very order, so the weights stay where they are; V^T's operand needs one channel of 8 tokens per lane: a lane loads d / 16 channels of
// those 8 rows (16 lanes one row, all of it) and regroups them with byte permutes, register to register.
//
// Bound by HBM: what is fetched is the rows' own size (414 of 420 MB).  4 x 8 heads of at most 32768 bf16 rows 83 us with the join, 5.1 TB/s; equal
// lengths 5.4, sixteen sequences of them 5.9; 32 x 8 heads of at most 8192 8-bit rows 76 us, 4.7 TB/s.  Of 1025 rows, 8 heads, 10 us: two launches.
#include "attend.h"
#include "mfma_util.h"
#include "wave_util.h"

namespace obc {
namespace {

using mfma::bf16x8;
using mfma::f32x4;

constexpr int kThreads = 256, kWaves = 4;

typedef const __attribute__((address_space(4))) int32_t *table_ptr;    // read through scalar loads

// What a wave has in flight or in hand of 32 tokens: rows as they lie in the cache.
template <int kD, bool kCodes>
struct Keys {
    static constexpr int kLoads = kCodes ? kD / 64 : kD / 32;           // 16-byte loads per block of 16 tokens
    u32x4 x[2][kLoads];
    uint32_t scale[2];
};
template <int kD, bool kCodes>
struct Values {
    static constexpr int kWords = kD * (kCodes ? 1 : 2) / 64;           // 32-bit words of d / 16 channels
    uint32_t x[8][kWords];
    u32x4 scale[2];                                                     // the scale bytes of four tokens each
};

// Workgroup of four waves: rows of one tile (at most 16 kSets), a share of the sequence, 32 tokens per wave in turn.
template <int kD, int kSets, bool kCodes>
__global__ __launch_bounds__(kThreads, 2) void attend_token(AttendArgs a, AttendPlan plan, float2 *part_ml, float *part_o) {
    constexpr int kSize = kCodes ? 1 : 2, kRow = kD * kSize, kSteps = kD / 32, kE = kD / 16, kScales = kD / kScaleBlock;
    constexpr int kPad = kD + 4;
    using K = Keys<kD, kCodes>;
    using V = Values<kD, kCodes>;
    __shared__ __attribute__((aligned(16))) float o_s[kWaves][16 * kSets][kPad];
    __shared__ float2 ml_s[kWaves][16 * kSets];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;
    const int split = blockIdx.x % plan.splits, bg = blockIdx.x / plan.splits;
    const Tile x = tile_of(a, bg, 0, plan.tile_rows);
    const int share = share_of(x.seen, plan);
    const int begin = split * share, end = min(begin + share, x.seen);
    if (begin >= end && split > 0) return;
    const CacheView &c = a.cache;

    // Queries as the second operand: row l % 16, the channels that the keys' load k of this lane brings.
    int seen[kSets];
    bf16x8 q[kSets][kSteps];
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
        const int row = 16 * s + col, t = row / a.G, h = x.g * a.G + row % a.G;
        const bool exists = t < a.T;
        seen[s] = exists ? min(x.sees(t, a.causal), end) : 0;
        const char *p = a.q + (((size_t)x.b * a.Hq + (exists ? h : x.g * a.G)) * a.T + (exists ? t : 0)) * (2 * kD);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int ch = kCodes ? 64 * (k / 2) + 16 * quad + 8 * (k % 2) : 32 * k + 8 * quad;
            q[s][k] = *(const bf16x8 *)(p + 2 * ch);
        }
    }
    const int full = x.n > 0 ? min(x.sees(0, a.causal), end) : 0;     // tokens that every row that counts sees

    f32x4 o[kSets][kE];
    float top[kSets], sum[kSets];
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
        top[s] = kNone;
        sum[s] = 0.f;
#pragma unroll
        for (int e = 0; e < kE; ++e) o[s][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // 16 consecutive rows lie in one page where pages hold at least 16 (shares begin at multiples of 32); a page is then looked up by a
    // scalar load.  (Four tokens' scale bytes are one load there, which an unpaged cache of odd length does not align.)  Rows past the end:
    // the last one again.
    const bool by_page = c.table ? c.page_size >= 16 : !kCodes || c.page_size % 4 == 0;
    const auto row_of = [&](int t) {
        const int j = min(t, end - 1);
        return row_in_pool(c, page_of(c, x.b, j), x.g, j);
    };
    const auto block_row = [&](int t) {            // of a block that lies in one page
        int page = x.b;
        if (c.table) page = ((table_ptr)(uintptr_t)(c.table + (size_t)x.b * c.pages_per_seq))[t >> c.shift];
        return row_in_pool(c, min(max(page, 0), c.num_pages - 1), x.g, t);
    };
    K kk;
    V vv;
    const auto load_keys = [&](int t0) {
        if (by_page && t0 + 32 <= end) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const size_t row = block_row(t0 + 16 * h);
                const char *p = c.k + row * kRow;
#pragma unroll
                for (int i = 0; i < K::kLoads; ++i) kk.x[h][i] = *(const u32x4 *)(p + (uint32_t)(col * kRow + 16 * quad + 64 * i));
                if constexpr (kCodes) kk.scale[h] = kScales == 4 ? *(const uint32_t *)(c.k_scale + row * 4 + (uint32_t)(col * 4))
                                                                 : *(const uint16_t *)(c.k_scale + row * 2 + (uint32_t)(col * 2));
            }
            return;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const size_t row = row_of(t0 + 16 * h + col);
#pragma unroll
            for (int i = 0; i < K::kLoads; ++i) kk.x[h][i] = *(const u32x4 *)(c.k + row * kRow + 16 * quad + 64 * i);
            if constexpr (kCodes) kk.scale[h] = kScales == 4 ? *(const uint32_t *)(c.k_scale + row * 4) : *(const uint16_t *)(c.k_scale + row * 2);
        }
    };
    const auto load_values = [&](int t0) {
        if (by_page && t0 + 32 <= end) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const size_t row = block_row(t0 + 16 * h);
                const char *p = c.v + row * kRow;
#pragma unroll
                for (int i = 0; i < 4; ++i) load_bytes<4 * V::kWords>(vv.x[4 * h + i], p + (uint32_t)(4 * quad * kRow + col * 4 * V::kWords + i * kRow));
                if constexpr (kCodes) {
                    if constexpr (kScales == 4) {
                        vv.scale[h] = *(const u32x4 *)(c.v_scale + row * 4 + (uint32_t)(16 * quad));
                    } else {
                        const u32x2 w = *(const u32x2 *)(c.v_scale + row * 2 + (uint32_t)(8 * quad));
                        vv.scale[h] = u32x4{w[0] & 0xffffu, w[0] >> 16, w[1] & 0xffffu, w[1] >> 16};
                    }
                }
            }
            return;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const size_t row = row_of(t0 + 16 * h + 4 * quad + i);
                load_bytes<4 * V::kWords>(vv.x[4 * h + i], c.v + row * kRow + col * 4 * V::kWords);
                if constexpr (kCodes) vv.scale[h][i] = kScales == 4 ? *(const uint32_t *)(c.v_scale + row * 4) : *(const uint16_t *)(c.v_scale + row * 2);
            }
    };

    const int first = begin + 32 * wave;
    if (first < end) {
        load_keys(first);
        load_values(first);
    }
    for (int t0 = first; t0 < end; t0 += 32 * kWaves) {
        const bool more = t0 + 32 * kWaves < end;
        f32x4 z[kSets][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int s = 0; s < kSets; ++s) z[s][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                bf16x8 kb;
                if constexpr (kCodes) {
                    const float scale = scale_value((kk.scale[h] >> (8 * (2 * (k / 2) + quad / 2))) & 0xffu);
                    const u32x2 lo = e4m3_bf16(kk.x[h][k / 2][2 * (k % 2)], scale), hi = e4m3_bf16(kk.x[h][k / 2][2 * (k % 2) + 1], scale);
                    kb = __builtin_bit_cast(bf16x8, (u32x4){lo[0], lo[1], hi[0], hi[1]});
                } else {
                    kb = __builtin_bit_cast(bf16x8, kk.x[h][k]);
                }
#pragma unroll
                for (int s = 0; s < kSets; ++s) z[s][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, q[s][k], z[s][h], 0, 0, 0);
            }
        }
        if (more) load_keys(t0 + 32 * kWaves);
        bf16x8 w[kSets];
#pragma unroll
        for (int s = 0; s < kSets; ++s) {
            if (t0 + 32 > full) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[s][h][r] = t0 + 16 * h + 4 * quad + r < seen[s] ? z[s][h][r] : -__builtin_inff();
            }
            float most = fmaxf(fmaxf(fmaxf(z[s][0][0], z[s][0][1]), fmaxf(z[s][0][2], z[s][0][3])),
                               fmaxf(fmaxf(z[s][1][0], z[s][1][1]), fmaxf(z[s][1][2], z[s][1][3])));
            most = across_rows<MaxOp>(most) * a.scale_log2;
            if (__any(most > top[s])) {
                const float now = fmaxf(top[s], most + kLazy), shrink = __builtin_amdgcn_exp2f(top[s] - now);
                top[s] = now;
                sum[s] *= shrink;
#pragma unroll
                for (int e = 0; e < kE; ++e) o[s][e] *= shrink;
            }
            const mfma::bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
            u32x4 p;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float e = __builtin_amdgcn_exp2f(fmaf(z[s][j / 2][2 * (j % 2)], a.scale_log2, -top[s]));
                const float f = __builtin_amdgcn_exp2f(fmaf(z[s][j / 2][2 * (j % 2) + 1], a.scale_log2, -top[s]));
                p[j] = mfma::pack_bf16(e, f);
                sum[s] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(mfma::bf16x2, (uint32_t)p[j]), one, sum[s], false);
            }
            w[s] = __builtin_bit_cast(bf16x8, p);
        }
        // V^T: of 8 tokens' words, the same half of each
        uint32_t words[8][kE / 2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (kCodes) {
                const float scale = scale_value((vv.scale[i / 4][i % 4] >> (8 * (col * kE / kScaleBlock))) & 0xffu);
#pragma unroll
                for (int j = 0; j < V::kWords; ++j) {
                    const u32x2 y = e4m3_bf16(vv.x[i][j], scale);
                    words[i][2 * j] = y[0];
                    words[i][2 * j + 1] = y[1];
                }
            } else {
#pragma unroll
                for (int j = 0; j < V::kWords; ++j) words[i][j] = vv.x[i][j];
            }
        }
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            u32x4 vb;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                vb[j] = __builtin_amdgcn_perm(words[2 * j + 1][e / 2], words[2 * j][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int s = 0; s < kSets; ++s) o[s][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vb), w[s], o[s][e], 0, 0, 0);
        }
        if (more) load_values(t0 + 32 * kWaves);
    }

    // The waves' sums, on the largest of their references.
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
        const float both = across_rows<SumOp>(sum[s]);
        const bool sees = seen[s] > 0;
        if (!sees) top[s] = kNone;
        if (quad == 0) ml_s[wave][16 * s + col] = make_float2(top[s], sees ? both : 0.f);
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
        float most = kNone;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, ml_s[w][16 * s + col].x);
        const float by = __builtin_amdgcn_exp2f(top[s] - most);
        const bool sees = seen[s] > 0;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < kE; e += 4) {
                const float4 y = make_float4(o[s][e][r] * by, o[s][e + 1][r] * by, o[s][e + 2][r] * by, o[s][e + 3][r] * by);
                *(float4 *)&o_s[wave][16 * s + col][kE * (4 * quad + r) + e] = sees ? y : make_float4(0.f, 0.f, 0.f, 0.f);
            }
    }
    __syncthreads();
    const int rows = a.G * a.T;
    for (int i = threadIdx.x; i < rows * (kD / 4); i += kThreads) {
        const int row = i / (kD / 4), ch = i % (kD / 4) * 4;
        float most = kNone, total = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, ml_s[w][row].x);
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float4 part = *(const float4 *)&o_s[w][row][ch];
            total += ml_s[w][row].y * __builtin_amdgcn_exp2f(ml_s[w][row].x - most);
            y.x += part.x; y.y += part.y; y.z += part.z; y.w += part.w;
        }
        if (plan.splits == 1) {
            const float inv = total > 0.f ? 1.f / total : 0.f;
            const float out[4] = {y.x * inv, y.y * inv, y.z * inv, y.w * inv};
            const int t = row / a.G, h = x.g * a.G + row % a.G;
            store4<OBC_BF16>(a.out + ((((size_t)x.b * a.T + t) * a.Hq + h) * kD + ch) * 2, out);
        } else {
            const size_t rec = ((size_t)split * a.B * a.Hkv + bg) * rows + row;
            if (ch == 0) part_ml[rec] = make_float2(most, total);
            *(float4 *)(part_o + rec * kD + ch) = y;
        }
    }
}

}  // namespace

hipError_t launch_attend_token(const AttendArgs &a, const AttendPlan &p, float2 *part_ml, float *part_o, hipStream_t stream) {
    const dim3 grid((unsigned)(a.B * a.Hkv * p.splits));
    using std::integral_constant;
    return with_types(a.d, a.dtype, a.cache_dtype, [&](auto dim, auto, auto codes) {
        if (p.tile_rows == 16) attend_token<dim.value, 1, codes.value><<<grid, kThreads, 0, stream>>>(a, p, part_ml, part_o);
        else attend_token<dim.value, 2, codes.value><<<grid, kThreads, 0, stream>>>(a, p, part_ml, part_o);
        return hipGetLastError();
    });
}

}  // namespace obc
