// Attention of new tokens over the cache: out = softmax(scale q k^T) v over the rows a token may see.
#include "attend.h"
#include "mfma_util.h"
#include "wave_util.h"

namespace obc {
namespace {

using mfma::f32x16;

// The general kernel, in fp32: one wave per (tile of 32 rows, share).  S^T = K Q^T and O^T = V^T P^T on the fp32 matrix cores: a
// lane holds one row's column of both, so the softmax needs one exchange between the wave's halves and no shuffle of P:
// register 4 j + i of S^T is token 8 j + 4 half + i, and as long as V's operand takes its tokens in that order the product is the same.
template <int kD, int kDtype, bool kCodes>
__global__ __launch_bounds__(256) void attend_plain(AttendArgs a, AttendPlan plan, float2 *part_ml, float *part_o) {
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int units = plan.tiles * plan.splits * a.B * a.Hkv;
    const int unit = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= units) return;
    const int split = unit % plan.splits, tile = unit / plan.splits % plan.tiles, bg = unit / (plan.splits * plan.tiles);
    const Tile x = tile_of(a, bg, tile * 32, 32);
    const int share = share_of(x.seen, plan.splits, plan.min_share);
    const int begin = split * share, end = min(begin + share, x.seen);
    if (begin >= end && split > 0) return;

    constexpr int kSize = kDtype == OBC_BF16 ? 2 : 4;
    const int row = x.r0 + col, t = row / a.G, h = x.g * a.G + row % a.G;
    const bool exists = t < a.T;
    const int seen = exists ? tokens_seen(x.len, x.n, t, a.causal) : 0;
    float q[kD / 2];             // channels 8 s + 4 half + i
    const char *q_row = a.q + (((size_t)x.b * a.Hq + (exists ? h : x.g * a.G)) * a.T + (exists ? t : 0)) * (kD * kSize);
#pragma unroll
    for (int s = 0; s < kD / 8; ++s) {
        const char *p = q_row + (8 * s + 4 * half) * kSize;
        if constexpr (kDtype == OBC_BF16) {
            const u32x2 w = *(const u32x2 *)p;
            q[4 * s] = __uint_as_float(w[0] << 16); q[4 * s + 1] = __uint_as_float(w[0] & 0xffff0000u);
            q[4 * s + 2] = __uint_as_float(w[1] << 16); q[4 * s + 3] = __uint_as_float(w[1] & 0xffff0000u);
        } else {
            *(float4 *)(q + 4 * s) = *(const float4 *)p;
        }
    }
    f32x16 o[kD / 32];
#pragma unroll
    for (int cb = 0; cb < kD / 32; ++cb) o[cb] = mfma::zero16();
    float top = kNone, sum = 0.f;

    for (int t0 = begin; t0 < end; t0 += 32) {
        const int kt = min(t0 + col, end - 1);                       // (rows past the share's end: its last one again, weight 0)
        const size_t krow = row_in_pool(a.cache, page_of(a.cache, x.b, kt), x.g, kt);
        f32x16 z = mfma::zero16();
#pragma unroll
        for (int s = 0; s < kD / 8; ++s) {
            float k[4];
            const int lo = 8 * s + 4 * half;
            if constexpr (kCodes) {
                e4m3_values(*(const uint32_t *)(a.cache.k + krow * kD + lo), scale_value(a.cache.k_scale[krow * (kD / kScaleBlock) + s / 4]), k);
            } else if constexpr (kDtype == OBC_BF16) {
                const u32x2 w = *(const u32x2 *)(a.cache.k + krow * (kD * 2) + lo * 2);
                k[0] = __uint_as_float(w[0] << 16); k[1] = __uint_as_float(w[0] & 0xffff0000u);
                k[2] = __uint_as_float(w[1] << 16); k[3] = __uint_as_float(w[1] & 0xffff0000u);
            } else {
                *(float4 *)k = *(const float4 *)(a.cache.k + krow * (kD * 4) + lo * 4);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) z = __builtin_amdgcn_mfma_f32_32x32x2f32(k[i], q[4 * s + i], z, 0, 0, 0);
        }
        float most = kNone;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int tok = t0 + 8 * (r / 4) + 4 * half + r % 4;
            z[r] = tok < min(seen, end) ? z[r] * a.scale_log2 : -__builtin_inff();
            most = fmaxf(most, z[r]);
        }
        const float now = fmaxf(top, mfma::halves_max(most));
        const float shrink = __builtin_amdgcn_exp2f(top - now);
        top = now;
        sum *= shrink;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            z[r] = __builtin_amdgcn_exp2f(z[r] - now);
            sum += z[r];
        }
#pragma unroll
        for (int cb = 0; cb < kD / 32; ++cb)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[cb][r] *= shrink;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int vt = min(t0 + 8 * (r / 4) + 4 * half + r % 4, end - 1);
            const size_t vrow = row_in_pool(a.cache, page_of(a.cache, x.b, vt), x.g, vt);
#pragma unroll
            for (int cb = 0; cb < kD / 32; ++cb) {
                float v;
                const int ch = 32 * cb + col;
                if constexpr (kCodes) {
                    const uint32_t code = *(const uint8_t *)(a.cache.v + vrow * kD + ch);
                    v = __builtin_amdgcn_cvt_f32_fp8((int)code, 0) * scale_value(a.cache.v_scale[vrow * (kD / kScaleBlock) + cb]);
                } else if constexpr (kDtype == OBC_BF16) {
                    v = bf16_bits_to_float(*(const uint16_t *)(a.cache.v + (vrow * kD + ch) * 2));
                } else {
                    v = *(const float *)(a.cache.v + (vrow * kD + ch) * 4);
                }
                o[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, z[r], o[cb], 0, 0, 0);
            }
        }
    }
    sum = mfma::halves_sum(sum);
    if (!exists) return;
    if (plan.splits == 1) {
        const float inv = sum > 0.f ? 1.f / sum : 0.f;
        char *to = a.out + (((size_t)x.b * a.T + t) * a.Hq + h) * (kD * kSize);
#pragma unroll
        for (int cb = 0; cb < kD / 32; ++cb)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float y[4] = {o[cb][4 * j] * inv, o[cb][4 * j + 1] * inv, o[cb][4 * j + 2] * inv, o[cb][4 * j + 3] * inv};
                store4<kDtype>(to + (32 * cb + 8 * j + 4 * half) * kSize, y);
            }
        return;
    }
    const size_t rec = ((size_t)split * a.B * a.Hkv + bg) * ((size_t)a.G * a.T) + row;
    if (half == 0) part_ml[rec] = make_float2(top, sum);
#pragma unroll
    for (int cb = 0; cb < kD / 32; ++cb)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            *(float4 *)(part_o + rec * kD + 32 * cb + 8 * j + 4 * half) =
                make_float4(o[cb][4 * j], o[cb][4 * j + 1], o[cb][4 * j + 2], o[cb][4 * j + 3]);
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
    const Tile x = tile_of(a, bg, row / plan.tile_rows * plan.tile_rows, plan.tile_rows);
    const int share = share_of(x.seen, plan.splits, plan.min_share);
    const int shares = max((x.seen + share - 1) / share, 1);
    float top = kNone, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const auto add = [&](const float2 m, const float4 o) {
        const float now = fmaxf(top, m.x), old = __builtin_amdgcn_exp2f(top - now), w = __builtin_amdgcn_exp2f(m.x - now);
        top = now;
        sum = sum * old + m.y * w;
        acc.x = acc.x * old + o.x * w; acc.y = acc.y * old + o.y * w; acc.z = acc.z * old + o.z * w; acc.w = acc.w * old + o.w * w;
    };
    for (int s = kManyRows ? 0 : slot; s < shares; s += kManyRows ? 1 : kSlots) {
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

void plan_attend(int B, int T, int Hq, int Hkv, int d, int capacity, int dtype, int cache_dtype, AttendPlan *p) {
    const long long rows = (long long)Hq / Hkv * T, heads = (long long)B * Hkv;
    *p = {};
    long long want, least;              // workgroups (waves) that fill the chip, tokens of the shortest share
    if (dtype == OBC_BF16 && rows <= 32) {
        p->form = kAttendToken;
        p->tile_rows = rows <= 16 ? 16 : 32;
        p->min_share = 128;
        // (us, 512 and 1024 workgroups: 64 x 8 heads x 1000 rows 42.5 and 49.6, 8 heads x 131072 101 and 105, 32 x 8 heads x 8192 ragged rows of
        // 8 bits 70.9 and 72.5; shares of 128 and 256 tokens, 8 heads x 1025 8.4 and 9.8)
        want = 512;
        least = 128;
    } else if (dtype == OBC_BF16) {
        // Two workgroups per compute unit.  A share costs its sums' way through memory, and one of few blocks its start (us, 32/8 heads: 512 rows over
        // 8192 in one share 101, in two 81; 1024 rows of 1024 in one 26.8, in two 33.3; 512 of 512 in one 16.4, in two 24.9; 16 over 8192
        // in shares of 1024 34.0, of 512 21.5, of 256 18.5; 256 over 2048 in shares of 512 28.7, of 256 30.4).
        const long long units = heads * ((rows + kAttendChunkRows - 1) / kAttendChunkRows);
        p->form = kAttendChunk;
        p->tile_rows = kAttendChunkRows;
        p->min_share = 32;
        want = 512;
        least = units >= 256 ? 2048 : units >= 64 ? 512 : 256;
    } else {
        p->form = kAttendPlain;
        p->tile_rows = 32;
        p->min_share = 32;
        want = 2048;
        least = 128;
    }
    p->tiles = (int)((rows + p->tile_rows - 1) / p->tile_rows);
    p->splits = (int)std::max(1LL, std::min(want / (heads * p->tiles), (capacity + least - 1) / least));
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
        e = with_types(a.d, a.dtype, a.cache_dtype, [&](auto dim, auto type, auto codes) {
            const long long units = (long long)p.tiles * p.splits * a.B * a.Hkv;
            attend_plain<dim.value, type.value, codes.value><<<dim3((unsigned)((units + 3) / 4)), 256, 0, stream>>>(a, p, ml, o);
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
