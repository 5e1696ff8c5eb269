// Attention of new tokens over the cache: out = softmax(scale q k^T) v over the rows a token may see.
#include "attend.h"
#include "mfma_util.h"
#include "wave_util.h"

namespace obc {
namespace {

using mfma::f32x16;

// fp32 queries, everything in fp32: one wave per (tile of 32 rows, share).  S^T = K Q^T and O^T = V^T P^T on the fp32 matrix cores: a
// lane holds one row's column of both, so the softmax needs one exchange between the wave's halves and no shuffle of P:
// register 4 j + i of S^T is token 8 j + 4 half + i, and V's operand takes its tokens in that order, its lane l channels
// (d / 32) l .. of a row, which 32 lanes read whole.
//
// Bound by the matrix cores from 32 rows per KV head on (8192 cycles per 32 tokens, d = 128; one wave per SIMD, since queries, sums, and
// the keys and values of the next block take 256 registers), by the cache's way from memory below.  256 rows over 4096 tokens, 32/8 heads,
// 172 us, 97 TFLOP/s; single tokens of 4 x 8 heads x 8192 rows 55 us, 4.8 TB/s; 2 x 8 heads, 77 rows over 1500 tokens, d = 64, 20 us.
template <int kD, bool kCodes>
__global__ __launch_bounds__(256, 1) void attend_fp32(AttendArgs a, AttendPlan plan, float2 *part_ml, float *part_o) {
    constexpr int kE = kD / 32, kScales = kD / kScaleBlock, kRow = kCodes ? kD : 4 * kD;
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int units = plan.tiles * plan.splits * a.B * a.Hkv;
    const int unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= units) return;
    const int split = unit % plan.splits, tile = unit / plan.splits % plan.tiles, bg = unit / (plan.splits * plan.tiles);
    const Tile x = tile_of(a, bg, tile * 32, 32);
    const int share = share_of(x.seen, plan);
    const int begin = split * share, end = min(begin + share, x.seen);
    if (begin >= end && split > 0) return;

    const int row = x.r0 + col, t = row / a.G, h = x.g * a.G + row % a.G;
    const bool exists = t < a.T;
    const int seen = exists ? min(x.sees(t, a.causal), end) : 0;
    const int full = x.r0 / a.G < x.n ? min(x.sees(x.r0 / a.G, a.causal), end) : 0;
    float4 q[kD / 8];             // channels 8 s + 4 half ..
    const char *q_row = a.q + (((size_t)x.b * a.Hq + (exists ? h : x.g * a.G)) * a.T + (exists ? t : 0)) * (kD * 4) + 16 * half;
#pragma unroll
    for (int s = 0; s < kD / 8; ++s) q[s] = *(const float4 *)(q_row + 32 * s);
    f32x16 o[kE];
#pragma unroll
    for (int e = 0; e < kE; ++e) o[e] = mfma::zero16();
    float top = kNone, sum = 0.f;

    // A block's rows as they lie in the cache, one block ahead; lane l (and l + 32) knows where row l % 32 of a block lies.  Rows past
    // the end: the last one again, with weight 0.
    const auto row_of = [&](int t0) -> unsigned long long {
        const int j = min(t0 + col, end - 1);
        return row_in_pool(a.cache, page_of(a.cache, x.b, j), x.g, j);
    };
    float4 k[kCodes ? 1 : kD / 8];
    uint32_t k8[kCodes ? kD / 8 : 1], k_scale = 0;
    float v[kCodes ? 1 : 16][kE];
    uint32_t v8[kCodes ? 16 : 1], v_scale[kCodes ? 16 : 1];
    const auto load_keys = [&](unsigned long long at) {
        const char *p = a.cache.k + at * kRow + (kCodes ? 4 : 16) * half;
#pragma unroll
        for (int s = 0; s < kD / 8; ++s) {
            if constexpr (kCodes) k8[s] = *(const uint32_t *)(p + 8 * s);
            else k[s] = *(const float4 *)(p + 32 * s);
        }
        if constexpr (kCodes) k_scale = kScales == 4 ? *(const uint32_t *)(a.cache.k_scale + at * 4) : *(const uint16_t *)(a.cache.k_scale + at * 2);
    };
    const auto load_values = [&](unsigned long long at) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const unsigned long long of = __shfl(at, 8 * (r / 4) + 4 * half + r % 4);
            const char *p = a.cache.v + of * kRow + kE * (kCodes ? 1 : 4) * col;
            if constexpr (!kCodes) load_bytes<4 * kE>(v[r], p);
            else v8[r] = kE == 4 ? *(const uint32_t *)p : *(const uint16_t *)p;
            if constexpr (kCodes) v_scale[r] = a.cache.v_scale[of * kScales + col * kE / kScaleBlock];
        }
    };

    unsigned long long next = 0;
    if (begin < end) {
        const unsigned long long at = row_of(begin);
        load_keys(at);
        load_values(at);
        next = row_of(begin + 32);
    }
    for (int t0 = begin; t0 < end; t0 += 32) {
        const bool more = t0 + 32 < end;
        f32x16 z = mfma::zero16();
#pragma unroll
        for (int s = 0; s < kD / 8; ++s) {
            float y[4];
            if constexpr (kCodes) e4m3_values(k8[s], scale_value((k_scale >> (8 * (s / 4))) & 0xffu), y);
            else y[0] = k[s].x, y[1] = k[s].y, y[2] = k[s].z, y[3] = k[s].w;
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(y[0], q[s].x, z, 0, 0, 0);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(y[1], q[s].y, z, 0, 0, 0);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(y[2], q[s].z, z, 0, 0, 0);
            z = __builtin_amdgcn_mfma_f32_32x32x2f32(y[3], q[s].w, z, 0, 0, 0);
        }
        if (more) load_keys(next);
        if (t0 + 32 > full) {
#pragma unroll
            for (int r = 0; r < 16; ++r) z[r] = t0 + 8 * (r / 4) + 4 * half + r % 4 < seen ? z[r] : -__builtin_inff();
        }
        float most = kNone;
#pragma unroll
        for (int r = 0; r < 16; ++r) most = fmaxf(most, z[r]);
        most = mfma::halves_max(most) * a.scale_log2;
        if (__any(most > top)) {
            const float now = fmaxf(top, most + kLazyFp32), shrink = __builtin_amdgcn_exp2f(top - now);
            top = now;
            sum *= shrink;
#pragma unroll
            for (int e = 0; e < kE; ++e) o[e] *= shrink;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            z[r] = __builtin_amdgcn_exp2f(fmaf(z[r], a.scale_log2, -top));
            sum += z[r];
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float y[4];
            if constexpr (kCodes) {
                e4m3_values(v8[r], scale_value(v_scale[r]), y);
            } else {
#pragma unroll
                for (int e = 0; e < kE; ++e) y[e] = v[r][e];
            }
#pragma unroll
            for (int e = 0; e < kE; ++e) o[e] = __builtin_amdgcn_mfma_f32_32x32x2f32(y[e], z[r], o[e], 0, 0, 0);
        }
        if (more) {
            load_values(next);
            next = row_of(t0 + 64);
        }
    }
    const bool sees = seen > 0, whole = plan.splits == 1;
    const float both = mfma::halves_sum(sum), total = sees ? both : 0.f, by = !sees ? 0.f : whole ? 1.f / total : 1.f;
    if (!exists) return;
    const size_t rec = ((size_t)split * a.B * a.Hkv + bg) * ((size_t)a.G * a.T) + row;
    if (!whole && half == 0) part_ml[rec] = make_float2(sees ? top : kNone, total);
    float *to = whole ? (float *)a.out + (((size_t)x.b * a.T + t) * a.Hq + h) * kD : part_o + rec * kD;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        float y[kE];
#pragma unroll
        for (int e = 0; e < kE; ++e) y[e] = sees ? o[e][r] * by : 0.f;
        float *p = to + kE * (8 * (r / 4) + 4 * half + r % 4);
        if constexpr (kE == 4) *(float4 *)p = make_float4(y[0], y[1], y[2], y[3]);
        else *(float2 *)p = make_float2(y[0], y[1]);
    }
}

// Joins the shares of a row: sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.  d / 4 lanes hold a row; a workgroup takes 256 / (d / 4) shares of one
// row at a time or, where rows have few shares, as many rows.
template <int kD, int kDtype, bool kManyRows>
__global__ __launch_bounds__(256) void attend_join(AttendArgs a, AttendPlan plan, const float2 *part_ml, const float *part_o) {
    constexpr int kLanes = kD / 4, kSlots = 256 / kLanes, kSize = kDtype == OBC_BF16 ? 2 : 4;
    const int rows = a.G * a.T, slot = threadIdx.x / kLanes, c = threadIdx.x % kLanes;
    const int at = kManyRows ? blockIdx.x * kSlots + slot : blockIdx.x;
    if (kManyRows && at >= a.B * a.Hkv * rows) return;
    const int bg = at / rows, row = at % rows;
    // The first record is on its way before the lengths say whether it counts: there is room for all of a plan's shares.
    const int first = kManyRows ? 0 : slot;
    const size_t rec_ahead = ((size_t)min(first, plan.splits - 1) * a.B * a.Hkv + bg) * rows + row;
    const float2 ml_ahead = part_ml[rec_ahead];
    const float4 o_ahead = *(const float4 *)(part_o + rec_ahead * kD + 4 * c);
    const Tile x = tile_of(a, bg, row / plan.tile_rows * plan.tile_rows, plan.tile_rows);
    const int share = share_of(x.seen, plan);
    const int shares = max((x.seen + share - 1) / share, 1);
    float top = kNone, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const auto add = [&](const float2 m, const float4 o) {
        const float now = fmaxf(top, m.x), old = __builtin_amdgcn_exp2f(top - now), w = __builtin_amdgcn_exp2f(m.x - now);
        top = now;
        sum = sum * old + m.y * w;
        acc.x = acc.x * old + o.x * w; acc.y = acc.y * old + o.y * w; acc.z = acc.z * old + o.z * w; acc.w = acc.w * old + o.w * w;
    };
    if (first < shares) add(ml_ahead, o_ahead);
    for (int s = first + (kManyRows ? 1 : kSlots); s < shares; s += kManyRows ? 1 : kSlots) {
        const size_t rec = ((size_t)s * a.B * a.Hkv + bg) * rows + row;
        add(part_ml[rec], *(const float4 *)(part_o + rec * kD + 4 * c));
    }
    if constexpr (!kManyRows) {
        __shared__ float4 sums[kSlots][kLanes];
        __shared__ float2 ml[kSlots];
        sums[slot][c] = acc;
        if (c == 0) ml[slot] = make_float2(top, sum);
        __syncthreads();
        if (slot != 0) return;
        for (int s = 1; s < min(kSlots, shares); ++s) add(ml[s], sums[s][c]);
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const int t = row / a.G, h = x.g * a.G + row % a.G;
    const float y[4] = {acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
    store4<kDtype>(a.out + ((((size_t)x.b * a.T + t) * a.Hq + h) * kD + 4 * c) * kSize, y);
}

size_t align_up(size_t x, size_t to) { return (x + to - 1) / to * to; }

}  // namespace

// Shares per tile for attend_chunk, by the time that a call of full length would take.  A block of 32 tokens takes a workgroup 0.79 us (d = 64:
// 0.54) alone on its compute unit and 1.05 (0.69) beside another; a round of workgroups starts in 4; joining takes 3 and its sums' way
// to memory and back.  Predicted / measured, us, 32/8 heads: 512 rows over 8192 tokens in two shares 116 / 98, in four 89 / 83; 1024 of 1024
// in one 29 / 27, in two 39 / 33; 256 over 2048 in four 27 / 29, in eight 30 / 30; four times 300 over 9000 in one 300 / 250, in three 235 / 217
// (of ragged lengths 226 and 143), in four 256 / 235; 64 over 32768 in 16 65 / 57, in 32 56 / 54.
// The lengths of a batch are not known here, and finer shares even out unlike ones: the mean of the time for full lengths and of one for lengths
// anywhere below (mean 1/2), whose workgroups take free places as they come.  Beyond 1024 tiles those even out by themselves.  Measured on random
// batches, 2 to 16 sequences of 7 head layouts, 16 to 2048 new rows over 512 to 32768.  By full lengths alone / by this rule, 12 batches where they
// differ: full lengths 0.97 (median; 0.86 to 1.03), half of them 0.90, random ones 1.12 (0.96 to 1.67), evenly spread 1.04, one full and the rest an eighth 1.55
// (0.91 to 2.56).  Mean 1/2 / 5/8, which 1 plan in 23 tells apart, 14 of those: full 1.02 (0.79 to 1.16), half 1.05, random 0.85, even 0.86, one long 0.65.
static int chunk_shares(long long units, long long rows, int d, int capacity, int batch) {
    const double alone = d == 128 ? 0.79 : 0.54, beside = d == 128 ? 1.05 : 0.69;
    const int blocks = (capacity + 31) / 32;
    int best = 1;
    double least = 0;
    for (int s = 1; s <= 64 && (s == 1 || blocks / s >= 4); ++s) {
        const long long n = units * s, left = n % 512;
        const double rounds = (double)(n / 512) * beside + (left == 0 ? 0 : left <= 256 ? alone : beside);
        const int share = (blocks + s - 1) / s;
        double run = rounds * share;
        if (batch > 1 && units <= 1024) {
            const double unlike = n <= 256 ? alone * share : beside * share * (n <= 512 ? 1.0 : std::max(1.0, 0.5 * (double)n / 512 + 0.5));
            run = (run + std::min(run, unlike)) / 2;
        }
        const double t = run + 4.0 * ((n + 511) / 512) + (s > 1 ? 3 + (double)rows * s * d * 1.8e-6 : 0);
        if (s == 1 || t < least) { least = t; best = s; }
        if (n > 4096) break;
    }
    return best;
}

void plan_attend(int B, int T, int Hq, int Hkv, int d, int capacity, int dtype, int cache_dtype, AttendPlan *p) {
    const long long rows = (long long)Hq / Hkv * T, heads = (long long)B * Hkv;
    *p = {};
    long long want = 1, least = 1;      // workgroups (waves) that fill the chip, tokens of the shortest share
    if (dtype == OBC_BF16 && rows <= 32) {
        p->form = kAttendToken;
        p->tile_rows = rows <= 16 ? 16 : 32;
        p->step = p->min_share = 128;
        // (us, 512 and 1024 workgroups: 64 x 8 heads x 1000 rows 42.5 and 49.6, 8 heads x 131072 101 and 105, 32 x 8 heads x 8192 ragged rows of
        // 8 bits 70.9 and 72.5; shares of 128 and 256 tokens, 8 heads x 1025 8.4 and 9.8.  One share needs no second launch: in shares and
        // in one 8 heads x 200 8.0 and 6.7, x 500 9.2 and 9.3, x 1025 8.6 and 14.6; 128 heads x 1025 19.1 and 17.7, x 2000 26.3 and 29.0;
        // 256 heads x 2000 43.5 and 42.7.)
        want = 512;
        least = capacity <= std::max(512LL, 10 * heads) ? capacity : 128;
    } else if (dtype == OBC_BF16) {
        p->form = kAttendChunk;
        p->tile_rows = kAttendChunkRows;
        p->step = 32;
        p->min_share = 128;
        p->tiles = (int)((rows + kAttendChunkRows - 1) / kAttendChunkRows);
        p->splits = chunk_shares(heads * p->tiles, heads * rows, d, capacity, B);
    } else {
        // One wave per SIMD, however short its share (us, 1024 waves and 2048: 4 x 8 heads x 8192 rows, G = 4, 55.5 and 64.1; 256 rows over 4096 172
        // and 185; shares of 32 and 128 tokens: 8 heads x 1000 rows 15.5 and 29.7).
        p->form = kAttendFp32;
        p->tile_rows = 32;
        p->step = p->min_share = 32;
        want = 1024;
        least = 32;
    }
    if (p->form != kAttendChunk) {
        p->tiles = (int)((rows + p->tile_rows - 1) / p->tile_rows);
        p->splits = (int)std::max(1LL, std::min(want / (heads * p->tiles), (capacity + least - 1) / least));
    }
    if (p->splits > 1) {
        const size_t records = (size_t)p->splits * heads * rows;
        p->part_ml = 0;
        p->part_o = align_up(records * sizeof(float2), 256);
        p->total = align_up(p->part_o + records * d * sizeof(float), 256);
    }
}

hipError_t launch_attend(const AttendArgs &a, const AttendPlan &p, char *workspace, hipStream_t stream) {
    float2 *ml = (float2 *)(workspace + p.part_ml);
    float *o = (float *)(workspace + p.part_o);
    hipError_t e = hipSuccess;
    if (p.form == kAttendChunk) {
        e = launch_attend_chunk(a, p, ml, o, stream);
    } else if (p.form == kAttendToken) {
        e = launch_attend_token(a, p, ml, o, stream);
    } else {
        e = with_types(a.d, a.dtype, a.cache_dtype, [&](auto dim, auto, auto codes) {
            const long long units = (long long)p.tiles * p.splits * a.B * a.Hkv;
            attend_fp32<dim.value, codes.value><<<dim3((unsigned)((units + 3) / 4)), 256, 0, stream>>>(a, p, ml, o);
            return hipGetLastError();
        });
    }
    if (e != hipSuccess || p.splits == 1) return e;
    return with_types(a.d, a.dtype, a.cache_dtype, [&](auto dim, auto type, auto) {
        const int rows = a.B * a.Hkv * a.G * a.T, per = 1024 / dim.value;
        if (p.splits <= 8) attend_join<dim.value, type.value, true><<<dim3((rows + per - 1) / per), 256, 0, stream>>>(a, p, ml, o);
        else attend_join<dim.value, type.value, false><<<dim3(rows), 256, 0, stream>>>(a, p, ml, o);
        return hipGetLastError();
    });
}

}  // namespace obc
