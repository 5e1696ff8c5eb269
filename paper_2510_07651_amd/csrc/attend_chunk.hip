// Attention of a chunk of bf16 queries over the cache, on the bf16 matrix cores.
#include "attend.h"
#include "mfma_util.h"
#include "wave_util.h"

namespace obc {
namespace {

using mfma::bf16x8;
using mfma::f32x16;
using mfma::i16x4;

constexpr int kThreads = 256, kTileRows = kAttendChunkRows;
constexpr int kRing = 4;               // blocks of 32 tokens in LDS

template <int kD>
struct Shape {
    static constexpr int kRow = 2 * kD, kPieces = kD / 8, kBlock = 32 * kRow, kSlot = 2 * kBlock;     // a slot: K block, V block
    static constexpr int kSteps = kD / 16, kCols = kD / 32;
};

// LDS blocks hold 32 rows of d bf16.  Row R keeps its 16-byte piece c at another slot, so that the reads meet no bank twice:
// keys are read one piece of 16 consecutive rows at a time, values 64 contiguous bytes of 4 consecutive rows.
template <int kD>
__device__ __forceinline__ int key_slot(int R, int c) { return kD == 128 ? c ^ (R & 15) : c ^ ((R >> 1) & 7); }
template <int kD>
__device__ __forceinline__ int value_slot(int R, int c) { return kD == 128 ? (c + 4 * (R & 3)) & 15 : (c + 4 * ((R >> 1) & 1)) & 7; }
template <int kD>
__device__ __forceinline__ int value_piece(int R, int slot) { return kD == 128 ? (slot - 4 * (R & 3)) & 15 : (slot - 4 * ((R >> 1) & 1)) & 7; }

// Groups that the eight dies are parted into, one per residue of the KV head.
__host__ __device__ constexpr int die_classes(int Hkv) { return Hkv % 8 == 0 ? 8 : Hkv % 4 == 0 ? 4 : Hkv % 2 == 0 ? 2 : 1; }

typedef const __attribute__((address_space(4))) int32_t *table_ptr;    // read through scalar loads

__device__ __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Brings blocks of 32 rows of K and V into LDS, block i of the share to slot i % kRing.  start(): block 0 is there after the next
// barrier, and of 8-bit rows block 1, with block 2 under way; of bf16 rows blocks 1 and 2 as well (the share's first three blocks are waited
// for together).  turn(i), by all waves: block i + 1 is there and block i - 1 may be overwritten; slice(0, i), slice(1, i): what is left to do
// of step i, between its first matrix ops.
template <int kD, bool kCodes>
struct Loader;

// bf16 rows go to LDS directly.  8 consecutive rows lie in one page where pages hold at least 8, and then the page is looked up by
// a scalar load, once for the wave.
template <int kD>
struct Loader<kD, false> {
    using S = Shape<kD>;
    static constexpr int kRowsPer = 1024 / S::kRow, kParts = 8 / kRowsPer, kInFlight = 2 * kParts;   // transfers of a wave per block
    const CacheView &c;
    int b, g, begin, end, blocks, wave, lane;
    bool by_page;
    uint32_t off_k[kParts], off_v[kParts];
    uint32_t lds;

    __device__ Loader(const CacheView &cache, const Tile &x, int begin_, int end_, int wave_, int lane_, char *smem)
        : c(cache), b(x.b), g(x.g), begin(begin_), end(end_), blocks((end_ - begin_ + 31) / 32), wave(wave_), lane(lane_),
          by_page(!cache.table || cache.page_size >= 8), lds(mfma::lds_offset_of(smem)) {
#pragma unroll
        for (int n = 0; n < kParts; ++n) {
            const int R = wave * 8 + n * kRowsPer + lane / S::kPieces, slot = lane % S::kPieces;
            const int row = n * kRowsPer + lane / S::kPieces;
            off_k[n] = row * S::kRow + key_slot<kD>(R, slot) * 16;
            off_v[n] = row * S::kRow + value_piece<kD>(R, slot) * 16;
        }
    }
    __device__ void start() const {
#pragma unroll
        for (int i = 0; i < kRing - 1; ++i)
            if (i < blocks) issue(i);
        mfma::wait_async_loads();
    }
    __device__ void turn(int i) const {
        if (i + 2 < blocks) mfma::wait_async_loads_keep<kInFlight>();
        else mfma::wait_async_loads();
        barrier();
        if (i + 3 < blocks) issue(i + 3);
    }
    __device__ void slice(int, int) const {}
    __device__ void issue(int i) const {
        const int t = begin + 32 * i + wave * 8;
        const uint32_t to = lds + i % kRing * S::kSlot + wave * 8 * S::kRow;
        if (by_page && t + 7 < end) {
            int page = b;
            if (c.table) page = ((table_ptr)(uintptr_t)(c.table + (size_t)b * c.pages_per_seq))[t >> c.shift];
            page = min(max(page, 0), c.num_pages - 1);
            const size_t at = row_in_pool(c, page, g, t) * S::kRow;
#pragma unroll
            for (int n = 0; n < kParts; ++n) mfma::dma16_based<false>(c.k + at, off_k[n], to + n * 1024);
#pragma unroll
            for (int n = 0; n < kParts; ++n) mfma::dma16_based<false>(c.v + at, off_v[n], to + S::kBlock + n * 1024);
            return;
        }
#pragma unroll
        for (int n = 0; n < kParts; ++n) {
            const int row = n * kRowsPer + lane / S::kPieces;
            const int j = min(t + row, end - 1);                        // (rows past the end: the last one again)
            const size_t at = row_in_pool(c, page_of(c, b, j), g, j) * S::kRow;
            mfma::dma16<false>(c.k + at + (off_k[n] - row * S::kRow), to + n * 1024);
            mfma::dma16<false>(c.v + at + (off_v[n] - row * S::kRow), to + S::kBlock + n * 1024);
        }
    }
};

// 8-bit rows pass through registers: fetched a block ahead of when they are written to LDS as bf16, exactly (16 codes per thread
// and tensor; with d = 64 half of the threads bring the keys, half the values).
template <int kD>
struct Loader<kD, true> {
    using S = Shape<kD>;
    static constexpr int kPerRow = kD / 16, kRows = 64 / kPerRow, kTensors = kD == 128 ? 2 : 1, kScales = kD / kScaleBlock;
    const CacheView &c;
    int b, g, begin, end, first, lane;        // first: the wave's first row of a block
    bool by_page, values;
    char *smem;
    u32x4 x[kTensors];
    uint32_t scale[kTensors];

    __device__ Loader(const CacheView &cache, const Tile &tile, int begin_, int end_, int wave, int lane_, char *smem_)
        : c(cache), b(tile.b), g(tile.g), begin(begin_), end(end_), first(kTensors == 2 ? wave * kRows : wave % 2 * kRows), lane(lane_),
          by_page(!cache.table || cache.page_size >= kRows), values(kTensors == 1 && wave >= 2), smem(smem_) {}
    __device__ void start() {
        fetch(0);
        slice(0, -2);
        slice(1, -2);
        slice(0, -1);
        slice(1, -1);
    }
    __device__ void turn(int) const { barrier(); }
    __device__ void slice(int n, int i) {
        if (n < kTensors) stage(n, (i + 2) % kRing);
        if (n == 1) fetch(i + 3);
    }
    __device__ void fetch(int i) {            // (blocks past the end: its last row)
        const int t = begin + 32 * i + first, piece = lane % kPerRow;
        size_t row;
        if (by_page && t + kRows <= end) {
            int page = b;
            if (c.table) page = ((table_ptr)(uintptr_t)(c.table + (size_t)b * c.pages_per_seq))[t >> c.shift];
            row = row_in_pool(c, min(max(page, 0), c.num_pages - 1), g, t) + lane / kPerRow;
        } else {
            const int j = min(t + lane / kPerRow, end - 1);
            row = row_in_pool(c, page_of(c, b, j), g, j);
        }
#pragma unroll
        for (int n = 0; n < kTensors; ++n) {
            const bool v = kTensors == 2 ? n == 1 : values;
            x[n] = *(const u32x4 *)((v ? c.v : c.k) + row * kD + piece * 16);
            scale[n] = (v ? c.v_scale : c.k_scale)[row * kScales + piece / 2];
        }
    }
    __device__ void stage(int n, int slot) const {
        const bool v = kTensors == 2 ? n == 1 : values;
        const int R = first + lane / kPerRow, piece = lane % kPerRow;
        const float by = scale_value(scale[n]);
        char *to = smem + slot * S::kSlot + (v ? S::kBlock : 0) + R * S::kRow;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u32x2 lo = e4m3_bf16(x[n][2 * h], by), hi = e4m3_bf16(x[n][2 * h + 1], by);
            const int at = v ? value_slot<kD>(R, 2 * piece + h) : key_slot<kD>(R, 2 * piece + h);
            *(u32x4 *)(to + at * 16) = u32x4{lo[0], lo[1], hi[0], hi[1]};
        }
    }
};

// Workgroup of four waves, 32 rows each, against a share of the sequence in blocks of 32 tokens.  S^T = K Q^T and O^T = V^T P^T: a lane
// holds one row's column of both, so the softmax needs one exchange between the wave's halves and no shuffle of P: register 4 j + i of
// S^T is token 8 j + 4 half + i, and V's operand takes its tokens in that order.
//
// Bound by matrix cores and vector ALUs in turn: 2048 rows over 16384 tokens, 32/8 heads, d = 128, 505 us, 1.02 PFLOP/s, on a card that held
// 2.08 GHz, 588 us on one that held 1.88; matrix cores busy 49 % of the cycles, vector ALUs 39 %, no bank conflicts.  Two workgroups share a compute unit, so one's vector work may run beside the other's
// matrix ops; 64 rows per wave with twice the registers reached 1.02, eight waves that share the ring 1.02.  8-bit rows, 2 x 509 rows over 20011
// tokens at most, 28/4 heads: 259 us, at the lower clock 287.
template <int kD, bool kCodes>
__global__ __launch_bounds__(kThreads, 2) void attend_chunk(AttendArgs a, AttendPlan plan, float2 *part_ml, float *part_o) {
    using S = Shape<kD>;
    __shared__ __attribute__((aligned(1024))) char smem[kRing * S::kSlot];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;

    // Which tile: workgroups go to the eight dies in turn; those of KV head g, of all sequences, stay on as few as there are KV heads for, so that
    // they find its rows in that die's L2 and every die has its part of the long sequences and of the short ones (us, with the dies dealt by
    // sequence and KV head, and so: 4 x 512 rows over at most 8192, 16/2 heads 155 and 124, 8 x 256, 8/1 heads 82 and 66; all of one length 170 and
    // 171, 94 and 95).  Late tiles, which see most, first (2048 rows of a prompt of 2048, 32/8 heads: 56.1 us, with those that share a
    // compute unit folded 50.9; 1500 over 4000 106.0, 103.7).
    const int heads = a.B * a.Hkv, die = blockIdx.x & 7, classes = die_classes(a.Hkv);
    const int per_head = plan.tiles * plan.splits, line = (per_head + 8 / classes - 1) / (8 / classes), mine = heads / classes;
    const int at = (int)(blockIdx.x >> 3);
    int head = at / line, in_line = at % line;
    if (mine * line <= 64) {                   // all at once, two per compute unit: the longest with the shortest
        const int j = at < 32 ? at : mine * line - 1 - (at - 32);
        head = j % mine;
        in_line = j / mine;
    }
    const int place = die / classes + 8 / classes * in_line, bg = die % classes + classes * head;
    if (place >= per_head) return;
    const int tile = plan.tiles - 1 - place / plan.splits, split = place % plan.splits;

    const Tile x = tile_of(a, bg, tile * kTileRows, kTileRows);
    const int share = share_of(x.seen, plan);
    const int begin = split * share, end = min(begin + share, x.seen), blocks = (end - begin + 31) / 32;
    if (blocks <= 0 && split > 0) return;

    const int r0 = x.r0 + wave * 32, row = r0 + col, t = row / a.G, h = x.g * a.G + row % a.G;
    const bool exists = t < a.T;
    const int seen = exists ? min(x.sees(t, a.causal), end) : 0;
    const int full = r0 / a.G < x.n ? min(x.sees(r0 / a.G, a.causal), end) : 0;    // tokens that every row that counts sees
    bf16x8 q[S::kSteps];
    const char *q_row = a.q + (((size_t)x.b * a.Hq + (exists ? h : x.g * a.G)) * a.T + (exists ? t : 0)) * S::kRow + half * 16;
#pragma unroll
    for (int k = 0; k < S::kSteps; ++k) q[k] = *(const bf16x8 *)(q_row + 32 * k);
    f32x16 o[S::kCols];
#pragma unroll
    for (int c = 0; c < S::kCols; ++c) o[c] = mfma::zero16();
    float top = kNone, sum = 0.f;
#pragma unroll
    for (int k = 0; k < S::kSteps; ++k) mfma::settle(q[k]);

    if (blocks > 0) {
        Loader<kD, kCodes> load(a.cache, x, begin, end, wave, lane, smem);
        int k_off[S::kSteps], v_off[S::kCols];
#pragma unroll
        for (int k = 0; k < S::kSteps; ++k) k_off[k] = col * S::kRow + key_slot<kD>(col, 2 * k + half) * 16;
#pragma unroll
        for (int c = 0; c < S::kCols; ++c) {
            const int i = lane & 15, sub = (lane >> 4) & 1, R = 4 * half + (i >> 2);
            v_off[c] = S::kBlock + R * S::kRow + value_slot<kD>(R, c * 4 + sub * 2 + ((i & 3) >> 1)) * 16 + (i & 1) * 8;
        }
        bf16x8 kb[S::kSteps], vb[2 * S::kCols];
        const auto read_keys = [&](int i) {
            const char *p = smem + (i % kRing) * S::kSlot;
#pragma unroll
            for (int k = 0; k < S::kSteps; ++k) kb[k] = mfma::lds_read16(p + k_off[k]);
        };
        const auto read_values = [&](int i) {
            const char *p = smem + (i % kRing) * S::kSlot;
#pragma unroll
            for (int j = 0; j < 2 * S::kCols; ++j) {
                union { bf16x8 v; i16x4 h[2]; } u;
                typedef __attribute__((address_space(3))) i16x4 *lds4;
                u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + v_off[j / 2] + 16 * (j % 2) * S::kRow));
                u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + v_off[j / 2] + (16 * (j % 2) + 8) * S::kRow));
                vb[j] = u.v;
            }
        };
        f32x16 z, z_next;
        union { uint32_t u[8]; bf16x8 v[2]; } w;
        const auto slot_end = [] { __builtin_amdgcn_sched_barrier(0); };
        const auto logit = [&](f32x16 &to, int k) { to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kb[k], q[k], to, 0, 0, 0); };
        const auto output = [&](int j) { o[j / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb[j], w.v[j % 2], o[j / 2], 0, 0, 0); };
        // Hides what a row does not see of block i; the largest logit that is left, in log2.
        const auto largest = [&](f32x16 &of, int i) {
            const int t0 = begin + 32 * i;
            if (t0 + 32 > full) {
#pragma unroll
                for (int r = 0; r < 16; ++r) of[r] = t0 + 8 * (r / 4) + 4 * half + r % 4 < seen ? of[r] : -__builtin_inff();
            }
            float most = mfma::max3(of[0], of[1], of[2]);
#pragma unroll
            for (int r = 3; r < 15; r += 2) most = mfma::max3(most, of[r], of[r + 1]);
            return mfma::halves_max(fmaxf(most, of[15])) * a.scale_log2;
        };
        // Moves the row's reference if a logit has outgrown it.
        const auto refer = [&](float most) {
            if (__any(most > top)) {
                const float now = fmaxf(top, most + kLazy), shrink = __builtin_amdgcn_exp2f(top - now);
                top = now;
                sum *= shrink;
#pragma unroll
                for (int c = 0; c < S::kCols; ++c) o[c] *= shrink;
            }
        };
        // Weights of the pairs from .. to - 1 of eight: two tokens each.  Their sum is taken of what they are rounded to.
        const mfma::bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
        const auto weigh = [&](int from, int to) {
#pragma unroll
            for (int j = from; j < to; ++j) {
                const float e = __builtin_amdgcn_exp2f(fmaf(z[2 * j], a.scale_log2, -top));
                const float f = __builtin_amdgcn_exp2f(fmaf(z[2 * j + 1], a.scale_log2, -top));
                w.u[j] = mfma::pack_bf16(e, f);
                sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(mfma::bf16x2, w.u[j]), one, sum, false);
            }
        };

        load.start();
        barrier();
        read_keys(0);
        read_values(0);
        z = mfma::zero16();
#pragma unroll
        for (int k = 0; k < S::kSteps; ++k) logit(z, k);
        float most = largest(z, 0);
        // Step i: the next block's logits beside this one's weights, one matrix op and a slice of vector work per slot, then this
        // block's outputs beside the largest of those logits.
        for (int i = 0; i + 1 < blocks; ++i) {
            load.turn(i);
            read_keys(i + 1);
            load.slice(0, i);
            load.slice(1, i);
            refer(most);
            slot_end();
            // (8-bit rows leave the vector ALUs more to do outside the slots: a wave inside them goes first.  2 x 509 rows over 20011 tokens, 28/4 heads:
            // 324 us without, 300 with; bf16 rows 497 us without, 516 with, 2048 rows over 16384.)
            if constexpr (kCodes) __builtin_amdgcn_s_setprio(1);
            z_next = mfma::zero16();
#pragma unroll
            for (int k = 0; k < S::kSteps; ++k) {
                logit(z_next, k);
                weigh(k * 8 / S::kSteps, (k + 1) * 8 / S::kSteps);
                slot_end();
            }
#pragma unroll
            for (int j = 0; j < S::kCols; ++j) output(j);
            slot_end();
            most = largest(z_next, i + 1);
#pragma unroll
            for (int j = S::kCols; j < 2 * S::kCols; ++j) output(j);
            if constexpr (kCodes) __builtin_amdgcn_s_setprio(0);
            z = z_next;
            read_values(i + 1);
        }
        refer(most);
        weigh(0, 8);
#pragma unroll
        for (int j = 0; j < 2 * S::kCols; ++j) output(j);
    }

    // (rows behind the chunk's end share a tile with rows that see something: what they have summed up is dropped here)
    const bool sees = seen > 0, whole = plan.splits == 1;
    const float both = mfma::halves_sum(sum), total = sees ? both : 0.f, by = !sees ? 0.f : whole ? 1.f / total : 1.f;
    if (!exists) return;
    const size_t rec = ((size_t)split * heads + bg) * ((size_t)a.G * a.T) + row;
    if (!whole && half == 0) part_ml[rec] = make_float2(sees ? top : kNone, total);
#pragma unroll
    for (int c = 0; c < S::kCols; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int ch = 32 * c + 8 * j + 4 * half;
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = sees ? o[c][4 * j + i] * by : 0.f;
            if (whole) store4<OBC_BF16>(a.out + ((((size_t)x.b * a.T + t) * a.Hq + h) * kD + ch) * 2, y);
            else store4<OBC_F32>(part_o + rec * kD + ch, y);
        }
}

}  // namespace

hipError_t launch_attend_chunk(const AttendArgs &a, const AttendPlan &p, float2 *part_ml, float *part_o, hipStream_t stream) {
    const int heads = a.B * a.Hkv, classes = die_classes(a.Hkv);
    const long long per_head = (long long)p.tiles * p.splits, line = (per_head + 8 / classes - 1) / (8 / classes);
    const dim3 grid((unsigned)(8 * line * (heads / classes)));
    return with_types(a.d, a.dtype, a.cache_dtype, [&](auto dim, auto, auto codes) {
        attend_chunk<dim.value, codes.value><<<grid, kThreads, 0, stream>>>(a, p, part_ml, part_o);
        return hipGetLastError();
    });
}

}  // namespace obc
