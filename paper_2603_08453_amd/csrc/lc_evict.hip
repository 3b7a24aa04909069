// Eviction of chunks by the attention weight that they have gathered: the weights (lc_weigh_chunks, lc_weigh_chunks4), whom to keep
// (lc_evict_select), the cache without the others (lc_evict_rows, lc_evict_rows4).
#include "lc_cache4.h"
#include "lc_internal.h"
#include "lc_select.h"

#include <type_traits>

#define LC_LOG2E 1.4426950408889634f
#define LC_LOG2E_REST 1.925963033500e-08f      // log2(e) less that
#define LC_INLINE __attribute__((always_inline))
#define LC_WG_THREADS 256
#define LC_WG_WAVES (LC_WG_THREADS / 64)
#define LC_WG_LONG 512            // tokens from which on a chunk is shared by the workgroup's wavefronts
#define LC_WG_ROWS 32             // tokens of a step
#define LC_WG_GROUPS 2048         // workgroups at most (rounded up to whole pairs)

namespace {

// ---------------------------------------------------------------- weights
// weights[chunk] += sum over its tokens t and the group's heads g of e^(q_g.k_t / sqrt(d) - lse_g), what the softmax with this log-sum-exp gives the
// chunk.  A listed chunk belongs to one wavefront (a long one to one workgroup) and is added up in a fixed order, so the result has the same bits
// every time.  The products are the attention's: 16 tokens are the rows of four 16x16x32 operands, the heads the columns.
struct LcWeighArgs {
    LcDev ix;
    const uint16_t* q;
    const void* K;
    long long seq, head;  // strides of K in bytes
    int tok;
    int max_tokens;
    const int32_t* ids;
    const int32_t* counts;
    int cap;
    const float* lse;     // [B][H*G]
    float* weights;       // [B][H][cap0]
    int G;                // heads of a group
};

//
// A workgroup has some entries of a list, whose chunks, boundaries and weights so far come in one go, a lane to an entry, 64 at a time; a wavefront takes every fourth of
// them and goes through their tokens 32 at a time, the next step's keys on their way, the next chunk's behind a chunk's last.
// Bound by the bytes for long lists, by the chain count, ids, boundaries, keys for short ones.  Every chunk of 4 x 32K tokens, 8 heads, 4 bits 18.8 us (71 MB, 3.8 TB/s), of
// 8 to 16 tokens 22; bfloat16 57 (268 MB, 4.7 TB/s); the 85 listed of 128K tokens 5.9 (bfloat16), 4.5 (4 bits).  A chunk to a wavefront, each with its own chain, took
// 25.9 us for the first and 6.9 for the last but one.  Group sizes are no variants: the products have 16 columns in any case.
template <bool IN4>
__global__ void __launch_bounds__(LC_WG_THREADS)
lc_weigh_kernel(const LcWeighArgs a) {
    lc_fetch_args<sizeof(LcWeighArgs)>();
    __shared__ float part_sh[LC_WG_WAVES];
    const LcDev& ix = a.ix;
    const int h = blockIdx.x, b = blockIdx.y, bh = b * ix.H + h, part = blockIdx.z, parts = gridDim.z;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, kg = lane >> 4;
    const int G = a.G, head = min(n, G - 1);
    // The entries are dealt evenly, a chunk to a wavefront at least.  How many there are the device knows alone (a list's table may have room for
    // far more): the first ones are on their way before the count is there, and the workgroups without entries are the last ones of all (as the last ones
    // of each pair they left the others on a few compute units: 12.0 us instead of 6.0 with room for 512 and more where 85 were listed).
    const __amdgpu_buffer_rsrc_t ids_r = lc_buffer(a.ids + (size_t)bh * a.cap, (int)(min((long long)a.cap, 1LL << 28) * 4));
    const int guess = part * LC_WG_WAVES;
    int id = lc_buf_load_i32(ids_r, guess + lane), before = lc_buf_load_i32(ids_r, max(0, guess + lane - 1));
    const int count = max(0, min(a.counts[bh], min(a.cap, 1 << 28))), M = ix.state[bh * 4 + 1];
    const int per = max(LC_WG_WAVES, (count + parts - 1) / parts);
    const int e_lo = part * per, e_hi = min(count, e_lo + per);
    if (e_lo >= e_hi) return;
    // the query block as in the attention (bfloat16 rows: lane (kg, n) has columns 8 kg + 32 j, 4-bit rows: 32 kg + 8 j)
    uint4 qb[4];
    {
        const uint16_t* qh = a.q + ((size_t)bh * G + head) * LC_D;
#pragma unroll
        for (int j = 0; j < 4; ++j) qb[j] = *reinterpret_cast<const uint4*>(qh + (IN4 ? 32 * kg + 8 * j : 8 * kg + 32 * j));
    }
    const float lse = a.lse[(size_t)bh * G + head];
    float* weights = a.weights + (size_t)bh * ix.cap[0];
    const int* bnd = ix.bounds + (size_t)b * (ix.cap[0] + 1);
    const float scale = 0.08838834764831845f * LC_LOG2E;
    const float off = -lse * LC_LOG2E;
    // What rounding has taken from off would be missing from each of the head's shares, all the same way: it is put back as a factor of their sum.  (Where it
    // could be large the share is 0 or the logits are out of float32's reach.)  Error of the weights against float64, every chunk of 4 x 32K tokens: 4.6e-8, without it 1.8e-7, in the same time.
    const float rest = fabsf(off) < 8388608.f ? __builtin_amdgcn_exp2f(fmaf(-lse, LC_LOG2E, -off) - lse * LC_LOG2E_REST) : 1.f;
    const bool counts_in = n < G && lse != LC_NEG_INF;       // (a head that attended to nothing adds nothing, whatever its logits are now)
    constexpr int ROW = IN4 ? LC_ROW4 : 2 * LC_D, HALVES = LC_WG_ROWS / 16, PIECES = IN4 ? 1 : 4;
    const int slab_bytes = (a.max_tokens - 1) * a.tok + ROW;
    const __amdgpu_buffer_rsrc_t Kr = lc_buffer(static_cast<const char*>(a.K) + (size_t)b * a.seq + (size_t)h * a.head, slab_bytes);

    struct Keys { lc_v4i k[HALVES][PIECES]; int s[HALVES]; };
    // rows r .. r + 31 (from `hi` on: zeros)
    auto load = [&](Keys& w, int r, int hi) LC_INLINE {
#pragma unroll
        for (int t = 0; t < HALVES; ++t) {
            const int row = r + 16 * t + n, o = row < hi ? (int)((uint32_t)row * (uint32_t)a.tok) + 16 * kg : slab_bytes;
#pragma unroll
            for (int j = 0; j < PIECES; ++j) w.k[t][j] = __builtin_amdgcn_raw_buffer_load_b128(Kr, o, 64 * j, 0);
            w.s[t] = IN4 ? lc_buf_load_u8(Kr, o + 64 - 15 * kg) : 0;
        }
    };
    auto shares = [&](const Keys& w, int r, int hi) LC_INLINE -> float {
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < HALVES; ++t) {
            if (t > 0 && r + 16 * t >= hi) break;            // (the same for the wavefront)
            lc_f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                lc_bf16x8 k;
                if constexpr (IN4) k = __builtin_bit_cast(lc_bf16x8, lc_unpack4((uint32_t)w.k[t][0][j], lc_scale4((uint32_t)w.s[t])));
                else k = __builtin_bit_cast(lc_bf16x8, w.k[t][j]);
                d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, __builtin_bit_cast(lc_bf16x8, qb[j]), d, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += r + 16 * t + 4 * kg + i < hi ? __builtin_amdgcn_exp2f(fmaf(d[i], scale, off)) : 0.f;
        }
        return sum;
    };
    auto total = [&](float sum) LC_INLINE -> float {
        sum = lc_sum16(counts_in ? sum * rest : 0.f);
        sum = lc_add_halves(sum, sum);
        return lc_add_rows(sum, sum);
    };

    for (int e0 = e_lo; e0 < e_hi; e0 += 64) {
        const int n_e = min(64, e_hi - e0);
        if (e0 != guess) {
            id = lc_buf_load_i32(ids_r, e0 + lane);
            before = lc_buf_load_i32(ids_r, max(0, e0 + lane - 1));
        }
        // (an entry that is no chunk, or no larger than a chunk right before it, is passed over: it has no tokens)
        const bool real = lane < n_e && id >= 0 && id < M && (e0 + lane == 0 || id > before || before >= M);
        const int at = real ? id : 0;
        const int begin = bnd[at], end = real ? min(bnd[at + 1], a.max_tokens) : begin;
        const float so_far = weights[at];
        const int begin_short = end - begin < LC_WG_LONG ? begin : end;      // long chunks are done behind the others
        // the wavefront's steps: entry, first row, the chunk's end
        struct Place { int e, r, hi; };
        auto settle = [&](Place& p) LC_INLINE {                    // from the beginning of an entry to one with tokens
            for (; p.e < n_e; p.e += LC_WG_WAVES) {
                p.r = lc_readlane(begin_short, p.e);
                p.hi = lc_readlane(end, p.e);
                if (p.r < p.hi) return;
            }
            p.r = p.hi = 0;
        };
        auto next = [&](const Place& p) LC_INLINE -> Place {
            Place q = {p.e, p.r + LC_WG_ROWS, p.hi};
            if (q.r >= q.hi) {
                q.e += LC_WG_WAVES;
                settle(q);
            }
            return q;
        };
        Place p = {wave, 0, 0};
        settle(p);
        float sum = 0.f;
        auto step = [&](const Keys& w, const Place& p, const Place& q) LC_INLINE {
            sum += shares(w, p.r, p.hi);
            if (q.e != p.e) {
                const float all = total(sum) + __int_as_float(lc_readlane(__float_as_int(so_far), p.e));
                const int chunk = lc_readlane(id, p.e);
                if (lane == 0) weights[chunk] = all;
                sum = 0.f;
            }
        };
        if (p.e < n_e) {
            Keys x, y;
            load(x, p.r, p.hi);
            for (;;) {
                const Place q = next(p);
                load(y, q.r, q.hi);
                __builtin_amdgcn_sched_barrier(0);
                step(x, p, q);
                if (q.e >= n_e) break;
                p = next(q);
                load(x, p.r, p.hi);
                __builtin_amdgcn_sched_barrier(0);
                step(y, q, p);
                if (p.e >= n_e) break;
            }
        }
        // long chunks: a step of each wavefront in turn
        unsigned long long longs = __ballot(begin_short != begin);
        while (longs != 0ull) {
            const int e = __ffsll((long long)longs) - 1;
            longs &= longs - 1ull;
            const int lo = lc_readlane(begin, e), hi = lc_readlane(end, e);
            float mine = 0.f;
            Keys x, y;
            load(x, lo + wave * LC_WG_ROWS, hi);
            for (int r = lo + wave * LC_WG_ROWS; r < hi; r += 2 * LC_WG_WAVES * LC_WG_ROWS) {
                load(y, r + LC_WG_WAVES * LC_WG_ROWS, hi);
                __builtin_amdgcn_sched_barrier(0);
                mine += shares(x, r, hi);
                load(x, r + 2 * LC_WG_WAVES * LC_WG_ROWS, hi);
                __builtin_amdgcn_sched_barrier(0);
                mine += shares(y, r + LC_WG_WAVES * LC_WG_ROWS, hi);
            }
            mine = total(mine);
            if (lane == 0) part_sh[wave] = mine;
            __syncthreads();
            const float all = (part_sh[0] + part_sh[1]) + (part_sh[2] + part_sh[3]);
            if (tid == 0) weights[lc_readlane(id, e)] = all + __int_as_float(lc_readlane(__float_as_int(so_far), e));
            __syncthreads();
        }
    }
}

template <bool IN4>
int launch_weigh(LcWeighArgs& a, hipStream_t stream) {
    const int pairs = a.ix.B * a.ix.H, all = (a.cap - 1) / LC_WG_WAVES + 1, fit = (LC_WG_GROUPS + pairs - 1) / pairs;
    hipLaunchKernelGGL((lc_weigh_kernel<IN4>), dim3(a.ix.H, a.ix.B, all < fit ? all : fit), dim3(LC_WG_THREADS), 0, stream, a);
    LC_HIP_CHECK(hipGetLastError());
    return LC_OK;
}

// ---------------------------------------------------------------- whom to keep
#define LC_EV_THREADS 1024
#define LC_EV_SUM 256             // chunks of a workgroup that sums weights
#define LC_EV_SLAB 4096           // chunks a workgroup takes at a time where several share a sequence
#define LC_EV_GROUPS 128          // of those workgroups at most
#define LC_EV_DIGIT 11
#define LC_EV_BINS (1 << LC_EV_DIGIT)
#define LC_EV_FEW 64              // chunks among which the cut is found by comparing each with each
#define LC_EV_FUSED_MAX 4096      // chunks up to which the selecting workgroup sums the weights itself (8192 of 8 heads: 14.1 us, summed by others 15.3; of 32: 21.1, 15.8)
#define LC_EV_SINGLE_MAX 14336    // chunks up to which a sequence has one workgroup (12288: 16.1 us, with several 21.3; 14000: 19.2, 22.4; 16384: 24.4, 21.6; 26 K: 43, 24)

// Order-preserving map of a double: larger weight, larger key; what is not a number comes last (key 0).  Pinned chunks have a key behind all of them.
#define LC_EV_PINNED 0xffffffffffffffffull
__device__ __forceinline__ unsigned long long lc_weight_key(double w) {
    if (!(w == w)) return 0ull;
    const unsigned long long u = (unsigned long long)__double_as_longlong(w + 0.0);
    return (u >> 63) ? ~u : (u | (1ull << 63));
}
// A chunk's weight summed over the heads, in 64 bits: the order of two chunks does not hang on the rounding of their sums.
__device__ __forceinline__ double lc_chunk_weight(const float* w, int H, int cap) {
    double sum = 0.0;
    int h = 0;
    for (; h + 4 <= H; h += 4) {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = w[(size_t)(h + i) * cap];
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += (double)x[i];
    }
    for (; h < H; ++h) sum += (double)w[(size_t)h * cap];
    return sum;
}

struct LcEvictArgs {
    LcDev ix;
    const float* weights;
    unsigned long long* keys;
    int32_t *ids, *bounds, *counts, *lens;
    int keep, recent, sink;
    int sums;             // workgroups of a sequence that have summed the weights
    int32_t* range;       // what they leave, sequences range_seq apart
    long long range_seq;
    int32_t* spare;       // where several workgroups share a sequence: 2 max_chunks for each
};
// spare: the digits' tokens, the cut, its chunks' number, the last that is kept, {chunks, tokens} that each workgroup keeps, the ranges of the keys, the chunks at the cut
enum { LC_EVS_CUT = LC_EV_BINS, LC_EVS_N = LC_EVS_CUT + 4, LC_EVS_LAST, LC_EVS_KEPT = LC_EVS_LAST + 3, LC_EVS_RANGE = LC_EVS_KEPT + 2 * LC_EV_GROUPS };

// Minimum or maximum over the wavefront, in lane 63 (DPP shifts; lanes without a source keep their own).
template <bool MAX>
__device__ __forceinline__ uint32_t lc_wave_extreme(uint32_t v) {
    auto step = [&](uint32_t x) LC_INLINE { v = MAX ? max(v, x) : min(v, x); };
    step((uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x111, 0xF, 0xF, false));   // row_shr:1
    step((uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x112, 0xF, 0xF, false));   // row_shr:2
    step((uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x114, 0xF, 0xF, false));   // row_shr:4
    step((uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x118, 0xF, 0xF, false));   // row_shr:8
    step((uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x142, 0xA, 0xF, false));   // row_bcast:15 -> rows 1, 3
    step((uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x143, 0xC, 0xF, false));   // row_bcast:31 -> rows 2, 3
    return v;
}

// Keys of many chunks, by many workgroups.  Each leaves the tokens of its chunks that are not pinned, and the smallest and the largest upper half of their keys.
__global__ void __launch_bounds__(LC_EV_SUM)
lc_evict_keys_kernel(const LcEvictArgs a) {
    lc_fetch_args<sizeof(LcEvictArgs)>();
    __shared__ uint32_t red_sh[3][LC_EV_SUM / 64];
    const LcDev& ix = a.ix;
    const int b = blockIdx.y, tid = threadIdx.x, M = min(ix.state[b * ix.H * 4 + 1], ix.cap[0]);
    const int* bnd = ix.bounds + (size_t)b * (ix.cap[0] + 1);
    const int last = bnd[M];
    if (a.spare) {
        int32_t* spare = a.spare + (size_t)b * 2 * ix.cap[0];
        for (int i = blockIdx.x * LC_EV_SUM + tid; i < LC_EV_BINS; i += gridDim.x * LC_EV_SUM) spare[i] = 0;
        if (blockIdx.x == 0 && tid == 0) spare[LC_EVS_N] = 0;
    }
    int tok = 0;
    uint32_t lo = 0xffffffffu, hi = 0u;
    for (int j = blockIdx.x * LC_EV_SUM + tid; j < M; j += gridDim.x * LC_EV_SUM) {
        const int begin = bnd[j], end = bnd[j + 1];
        unsigned long long k = lc_weight_key(lc_chunk_weight(a.weights + (size_t)b * ix.H * ix.cap[0] + j, ix.H, ix.cap[0]));
        if (begin < a.sink || end > last - a.recent) {
            k = LC_EV_PINNED;
        } else {
            tok += end - begin;
            lo = min(lo, (uint32_t)(k >> 32));
            hi = max(hi, (uint32_t)(k >> 32));
        }
        a.keys[(size_t)b * ix.cap[0] + j] = k;
    }
    lo = lc_wave_extreme<false>(lo);
    hi = lc_wave_extreme<true>(hi);
    tok = lc_wave_scan_incl(tok);
    if ((tid & 63) == 63) { red_sh[0][tid >> 6] = lo; red_sh[1][tid >> 6] = hi; red_sh[2][tid >> 6] = (uint32_t)tok; }
    __syncthreads();
    if (tid == 0) {
        int32_t* const out = a.range + b * a.range_seq + 3 * blockIdx.x;
        lo = min(min(red_sh[0][0], red_sh[0][1]), min(red_sh[0][2], red_sh[0][3]));
        hi = max(max(red_sh[1][0], red_sh[1][1]), max(red_sh[1][2], red_sh[1][3]));
        out[0] = (int32_t)lo;
        out[1] = (int32_t)hi;
        out[2] = (int32_t)((red_sh[2][0] + red_sh[2][1]) + (red_sh[2][2] + red_sh[2][3]));
    }
}

// A lane's part of what the workgroups of the keys have left.
__device__ __forceinline__ void lc_evict_range(const LcEvictArgs& a, int b, uint32_t& lo, uint32_t& hi, int& tok) {
    const int32_t* from = a.range + b * a.range_seq;
    for (int i = threadIdx.x & 63; i < a.sums; i += 64) {
        lo = min(lo, (uint32_t)from[3 * i]);
        hi = max(hi, (uint32_t)from[3 * i + 1]);
        tok += from[3 * i + 2];
    }
}

// ---- finding the cut
struct LcCutSh {
    int tok[LC_EV_BINS];
    unsigned long long key[LC_EV_FEW], last_key;
    int id[LC_EV_FEW], len[LC_EV_FEW], sum[LC_EV_FEW];
    int scan[2 * (LC_EV_THREADS / 64)], found[2], few, last_id;
};
// (a barrier must follow)
__device__ __forceinline__ void lc_cut_prepare(LcCutSh& sh) {
    for (int i = threadIdx.x; i < LC_EV_BINS; i += LC_EV_THREADS) sh.tok[i] = 0;
    if (threadIdx.x < LC_EV_FEW) sh.sum[threadIdx.x] = 0;
    if (threadIdx.x == 0) { sh.few = 0; sh.last_key = 0ull; sh.last_id = -1; }
}
// Keys of [base, base + 2^shift) are at the cut: of those the first `left` tokens' worth is kept, of larger ones all, of smaller ones none.
struct LcCut {
    unsigned long long base;
    int shift, left;      // (a shift of 64: before the first digit)
    __device__ __forceinline__ int next() const { return max(0, shift - LC_EV_DIGIT); }
    __device__ __forceinline__ bool digit(unsigned long long k, int* d) const {      // whether a key is at the cut, and its next digit
        const unsigned long long x = (k - base) >> next();
        *d = (int)x;
        return k != LC_EV_PINNED && x < 1ull << (shift - next());
    }
    __device__ __forceinline__ bool at(unsigned long long k) const { return k != LC_EV_PINNED && ((k - base) >> shift) == 0ull; }
    __device__ __forceinline__ bool above(unsigned long long k) const { return k == LC_EV_PINNED || (k >= base && !at(k)); }
};
// All keys from the smallest to the largest upper half (lo > hi: there is none).
__device__ __forceinline__ LcCut lc_cut_of(uint32_t lo, uint32_t hi, int left) {
    return {(unsigned long long)lo << 32, 32 + (lo < hi ? 32 - __clz((int)(hi - lo)) : 0), left};
}
// One digit less at the cut: the one at which the tokens from above (t1: of digit BINS - 1 - 2 thread, t0: of the one below) no longer fit.
__device__ __forceinline__ void lc_cut_digit(LcCutSh& sh, LcCut& cut, int t1, int t0, bool clear) {
    const int d1 = LC_EV_BINS - 1 - 2 * threadIdx.x;
    int total;
    const int before = lc_block_scan<LC_EV_THREADS>(t1 + t0, sh.scan, &total);
    if (before <= cut.left && before + t1 > cut.left) { sh.found[0] = d1; sh.found[1] = before; }
    else if (before + t1 <= cut.left && before + t1 + t0 > cut.left) { sh.found[0] = d1 - 1; sh.found[1] = before + t1; }
    if (clear) sh.tok[d1] = sh.tok[d1 - 1] = 0;
    __syncthreads();
    cut.base += (unsigned long long)sh.found[0] << cut.next();
    cut.left -= sh.found[1];
    cut.shift = cut.next();
}
// sh.last_key, sh.last_id: every chunk up to them in the order is kept.  each(f): f(chunk, tokens, key) of all chunks at the cut and perhaps others, sorted(j, &tokens):
// the key of chunk j < M.  listed: there may be few of them at the cut already.  More tokens are at the cut than are left.
template <typename Each, typename Sorted>
__device__ __forceinline__ void lc_cut_search(LcCutSh& sh, LcCut cut, bool listed, int M, Each each, Sorted sorted) {
    constexpr int NT = LC_EV_THREADS, NW = NT / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // the chunks at the cut, if they are few
    auto collect = [&]() LC_INLINE -> bool {
        each([&](int j, int n, unsigned long long k) LC_INLINE {
            if (cut.at(k)) {
                const int i = atomicAdd(&sh.few, 1);
                if (i < LC_EV_FEW) {
                    sh.key[i] = k;
                    sh.id[i] = j;
                    sh.len[i] = n;
                }
            }
        });
        __syncthreads();
        if (sh.few <= LC_EV_FEW) return true;
        __syncthreads();
        if (tid == 0) sh.few = 0;
        __syncthreads();
        return false;
    };
    bool few = listed && collect();
    while (cut.shift > 0 && !few) {
        each([&](int, int n, unsigned long long k) LC_INLINE {
            int d;
            if (cut.digit(k, &d)) atomicAdd(&sh.tok[d], n);
        });
        __syncthreads();
        const int d1 = LC_EV_BINS - 1 - 2 * tid, t1 = sh.tok[d1], t0 = sh.tok[d1 - 1];
        lc_cut_digit(sh, cut, t1, t0, true);
        few = collect();
    }
    if (__builtin_expect(few, 1)) {
        // a lane has a chunk at the cut, each wavefront some of those to compare it with
        const int n = sh.few;
        const unsigned long long k = lane < n ? sh.key[lane] : 0ull;
        const int id = lane < n ? sh.id[lane] : 0x7fffffff;
        int part = 0;
        for (int i = wave; i < n; i += NW) {
            const unsigned long long ki = sh.key[i];
            if (ki > k || (ki == k && sh.id[i] <= id)) part += sh.len[i];
        }
        if (lane < n && part != 0) atomicAdd(&sh.sum[lane], part);
        __syncthreads();
        if (wave == 0) {
            // (the sums of those that fit grow along the order: the last of them has the largest)
            const int sum = sh.sum[lane];
            const uint32_t mine = lane < n && sum <= cut.left ? (uint32_t)sum + 1u : 0u;
            const uint32_t most = (uint32_t)lc_readlane((int)lc_wave_extreme<true>(mine), 63);
            if (most == 0u) {
                if (lane == 0) sh.last_key = cut.base + ((1ull << cut.shift) - 1ull);    // none at the cut
            } else if (mine == most) {
                sh.last_key = k;
                sh.last_id = id;
            }
        }
    } else {
        // equal keys at the cut: the first of them
        int tied = 0;
        for (int j0 = 0; j0 < M; j0 += NT) {
            const int j = j0 + tid;
            int n = 0;
            if (j < M && sorted(j, &n) != cut.base) n = 0;
            int total;
            const int before = lc_block_scan<NT>(n, sh.scan, &total);
            if (n > 0 && before <= cut.left - tied - n) atomicMax(&sh.last_id, j);
            tied = min(tied + total, 1 << 30);
        }
        if (tid == 0) sh.last_key = cut.base;
    }
    __syncthreads();
}

// The kept ones of chunks [j, hi), from place n_keep and token n_tok on: a thread has four chunks in a row, a scan for LC_EV_SLAB of them.
template <typename Kept>
__device__ __forceinline__ void lc_evict_place(int j0, int hi, const int* bnd, int32_t* ids, int32_t* bounds, int* scan_sh, int& n_keep, int& n_tok, Kept keeps) {
    for (; j0 < hi; j0 += LC_EV_SLAB) {
        const int j = j0 + 4 * (int)threadIdx.x;
        int edge[5];
#pragma unroll
        for (int u = 0; u < 5; ++u) edge[u] = bnd[min(j + u, hi)];
        uint32_t kept = keeps(j, edge);
        int n = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) n += (kept >> u) & 1u ? edge[u + 1] - edge[u] : 0;
        int at, to, count, tokens;
        lc_block_scan2<LC_EV_THREADS>(__popc(kept), n, scan_sh, &at, &to, &count, &tokens);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if ((kept >> u) & 1u) {
                ids[n_keep + at] = j + u;
                bounds[n_keep + at] = n_tok + to;
                at += 1;
                to += edge[u + 1] - edge[u];
            }
        n_keep += count;
        n_tok += tokens;
    }
}

// One workgroup per sequence: the pinned chunks, and of the others the longest prefix by (key descending, id ascending) that fits.  The cut
// is found digit by digit of the keys' distance from the smallest: tokens per digit, then the digit at which their sum from above no longer fits,
// until few chunks are left at the cut (mostly after one digit) or all their keys are equal.  (Digits of the keys themselves begin with the
// exponent, whose few values put all LDS atomics on a few words.)
// A thread keeps C chunks, 1024 apart, in registers; chunks beyond (more than 12288, or an index that has grown since the launch was captured) are read where they are
// each time.
// What bounds it is a chain of barriers, LDS atomics and the first loads in one compute unit per sequence: 113 chunks 5.9 us, 4 sequences of 455 6.1, 4096 9.5, 10.9 K 15.7 with the
// weights' sums before it (4.5; up to 4096 chunks the selecting workgroup makes them, which saves a launch), 4 sequences of 12 K 16.6.  (With the pinned chunks in masks beside the
// keys, and the range of the keys found here instead of with the sums: 10.9 K 16.9; with the loops over chunks in memory between the others in the code: the first two 6.3 and 6.5.
// Equal weights are the slow case, and all of the figures are for weights that differ.  With four fifths of the chunks exactly 0 (never listed) and the cut above them 4 sequences of
// 455 take 5.9 us, 4096 12.6, 10.9 K 24; with the cut among them, where every digit's tokens meet in one word and the ties are scanned, 14, 40 and 86.
// Digits of the keys from the first bit in which they differ, ranks by a single wavefront and scans of 1024 chunks at a time: 9 us for the first.)
template <int C, bool FUSED>
__global__ void __launch_bounds__(LC_EV_THREADS)
lc_evict_select_kernel(const LcEvictArgs a) {
    lc_fetch_args<sizeof(LcEvictArgs)>();
    constexpr int NT = LC_EV_THREADS, NW = NT / 64;
    __shared__ LcCutSh sh;
    __shared__ uint32_t red_sh[3 * NW];
    __shared__ int slab_cnt[C * NW], slab_tok[C * NW];
    const LcDev& ix = a.ix;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int T = ix.state[b * ix.H * 4 + 0], M = min(ix.state[b * ix.H * 4 + 1], ix.cap[0]);
    const int* bnd = ix.bounds + (size_t)b * (ix.cap[0] + 1);
    const unsigned long long* keys = a.keys + (size_t)b * ix.cap[0];
    const float* weights = a.weights + (size_t)b * ix.H * ix.cap[0];
    int32_t* ids = a.ids + (size_t)b * ix.cap[0];
    const int last = bnd[M];
    auto key_of = [&](int j, int begin, int end) LC_INLINE -> unsigned long long {
        if constexpr (!FUSED) return keys[j];
        const unsigned long long k = lc_weight_key(lc_chunk_weight(weights + j, ix.H, ix.cap[0]));
        return begin < a.sink || end > last - a.recent ? LC_EV_PINNED : k;
    };

    unsigned long long key[C];
    int len[C];
    {
        // (no branch around a load: they are on their way together)
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int j = max(0, min(tid + c * NT, M - 1)), begin = bnd[j], end = bnd[j + 1];
            const bool real = tid + c * NT < M;
            const unsigned long long k = key_of(j, begin, end);
            key[c] = real ? k : LC_EV_PINNED;
            len[c] = real ? end - begin : 0;
        }
    }
    // f(chunk, its tokens, its key) of the chunks in registers, then of the others
    auto each = [&](auto f) LC_INLINE {
#pragma unroll
        for (int c = 0; c < C; ++c)
            f(tid + c * NT, len[c], key[c]);
        // (four at a time, their loads together)
        if (__builtin_expect(M > C * NT, 0)) {
            for (int j0 = C * NT + tid; j0 < M; j0 += 4 * NT) {
                int n[4];
                unsigned long long k[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int j = min(j0 + u * NT, M - 1), begin = bnd[j], end = bnd[j + 1];
                    n[u] = end - begin;
                    k[u] = key_of(j, begin, end);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (j0 + u * NT < M) f(j0 + u * NT, n[u], k[u]);
            }
        }
    };

    // tokens of those that are not pinned, the smallest and the largest of their keys (of the upper halves)
    int tok = 0;
    uint32_t lo = 0xffffffffu, hi = 0u;
    if constexpr (FUSED) {
        each([&](int, int n, unsigned long long k) LC_INLINE {
            const bool is = k != LC_EV_PINNED;
            tok += is ? n : 0;
            lo = min(lo, (uint32_t)(k >> 32));               // (a pinned one's: the largest there is)
            hi = max(hi, is ? (uint32_t)(k >> 32) : 0u);
        });
    } else {
        lc_evict_range(a, b, lo, hi, tok);
    }
    lc_cut_prepare(sh);
    lo = lc_wave_extreme<false>(lo);
    hi = lc_wave_extreme<true>(hi);
    tok = lc_wave_scan_incl(tok);
    if constexpr (FUSED) {
        if (lane == 63) { red_sh[wave] = lo; red_sh[NW + wave] = hi; red_sh[2 * NW + wave] = (uint32_t)tok; }
        __syncthreads();
        lo = lc_wave_extreme<false>(red_sh[lane & (NW - 1)]);
        hi = lc_wave_extreme<true>(red_sh[NW + (lane & (NW - 1))]);
        tok = lc_wave_scan_incl(lane < NW ? (int)red_sh[2 * NW + lane] : 0);
    } else {
        __syncthreads();                                     // (the counts above are zero)
    }
    lo = (uint32_t)lc_readlane((int)lo, 63);
    hi = (uint32_t)lc_readlane((int)hi, 63);
    const int others = lc_readlane(tok, 63);
    const int left = max(0, a.keep - (last - others));       // tokens for the others, behind the pinned ones
    const bool all = others <= left;
    if (!all)
        lc_cut_search(sh, lc_cut_of(lo, hi, left), false, M, each, [&](int j, int* n) LC_INLINE {
            const int begin = bnd[j], end = bnd[j + 1];
            *n = end - begin;
            return key_of(j, begin, end);
        });
    const unsigned long long last_key = all ? 0ull : sh.last_key;
    const int last_id = all ? 0x7fffffff : sh.last_id;
    auto keeps = [&](unsigned long long k, int j) LC_INLINE { return k > last_key || (k == last_key && j <= last_id); };   // (pinned ones too)

    // ids, boundaries, the rest of both lists
    int32_t* bounds = a.bounds + (size_t)b * (ix.cap[0] + 1);
    int n_keep = 0, n_tok = 0;
    {
        // the chunks in registers all at once: wavefronts' counts and tokens, then each its place
        uint32_t kept = 0u;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int j = tid + c * NT;
            const bool k = j < M && keeps(key[c], j);
            kept |= k ? 1u << c : 0u;
            const int n = k ? len[c] : 0, tokens = lc_wave_scan_incl(n), count = __popcll(__ballot(k));
            len[c] = tokens - n;                             // (from here on: tokens kept before it, of the wavefront)
            if (lane == 63) { slab_cnt[c * NW + wave] = count; slab_tok[c * NW + wave] = tokens; }
        }
        __syncthreads();
        if (wave == 0) {
            int cc = 0, tt = 0;
#pragma unroll
            for (int i = 0; i < (C * NW + 63) / 64; ++i) {
                const int x = i * 64 + lane;
                const int c = x < C * NW ? slab_cnt[x] : 0, t = x < C * NW ? slab_tok[x] : 0;
                const int ci = lc_wave_scan_incl(c), ti = lc_wave_scan_incl(t);
                if (x < C * NW) { slab_cnt[x] = cc + ci - c; slab_tok[x] = tt + ti - t; }
                cc += lc_readlane(ci, 63);
                tt += lc_readlane(ti, 63);
            }
            if (lane == 0) { sh.found[0] = cc; sh.found[1] = tt; }
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const bool k = (kept >> c) & 1u;
            const int i = slab_cnt[c * NW + wave] + __popcll(__ballot(k) & ((1ull << lane) - 1ull));
            if (k) {
                ids[i] = tid + c * NT;
                bounds[i] = slab_tok[c * NW + wave] + len[c];
            }
        }
        n_keep = sh.found[0];
        n_tok = sh.found[1];
    }
    if (__builtin_expect(M > C * NT, 0)) lc_evict_place(C * NT, M, bnd, ids, bounds, sh.scan, n_keep, n_tok, [&](int j, const int* edge) LC_INLINE {
        uint32_t kept = 0u;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            kept |= j + u < M && (all || keeps(key_of(min(j + u, M - 1), edge[u], edge[u + 1]), j + u)) ? 1u << u : 0u;
        return kept;
    });
    for (int i = n_keep + tid; i < ix.cap[0]; i += NT) {
        ids[i] = -1;
        bounds[i] = n_tok;
    }
    if (tid == 0) {
        bounds[ix.cap[0]] = n_tok;
        a.counts[b] = n_keep;
        if (a.lens) a.lens[b] = n_tok + max(0, T - last);
    }
}

// ---- many chunks: several workgroups to a sequence, each with a range of its chunks
// One alone reads the keys at what a compute unit gets from its L2, and several times.  Three launches behind the keys': the first digit's tokens, added up by all, and by
// the last one to arrive the cut; the chunks above it, counted, those at it, listed, and by the last one the rest of the search among them; ids and boundaries.
// Bound by the four launches, each a few trips to memory long: 26 K chunks 24 us (by one workgroup 43), 87 K 28 (142).  That is with weights that differ; with four fifths of
// them 0 and the cut above those 31 and 55, with the cut among them, which the last workgroup alone goes through, 421 and 1257.
struct LcSlab {
    int lo, hi;           // chunks of this workgroup
    int size;             // of each
    __device__ __forceinline__ LcSlab(int M, int part, int parts) {
        size = ((M + parts - 1) / parts + LC_EV_SLAB - 1) / LC_EV_SLAB * LC_EV_SLAB;
        lo = min(M, (int)min((long long)part * size, (long long)M));
        hi = min(M - lo, size) + lo;
    }
};
// f(chunk, tokens, key, whether there is one) of a workgroup's chunks, in any order, by whole wavefronts
template <typename F>
__device__ __forceinline__ void lc_slab_each(const LcSlab& slab, const int* bnd, const unsigned long long* keys, F f) {
    constexpr int U = LC_EV_SLAB / LC_EV_THREADS;
    for (int j0 = slab.lo; j0 < slab.hi; j0 += LC_EV_SLAB) {
        int n[U];
        unsigned long long k[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = min(j0 + u * LC_EV_THREADS + (int)threadIdx.x, slab.hi - 1);
            n[u] = bnd[j + 1] - bnd[j];
            k[u] = keys[j];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * LC_EV_THREADS + (int)threadIdx.x;
            f(j, n[u], k[u], j < slab.hi);
        }
    }
}

__global__ void __launch_bounds__(LC_EV_THREADS)
lc_evict_cut_kernel(const LcEvictArgs a) {
    lc_fetch_args<sizeof(LcEvictArgs)>();
    __shared__ LcCutSh sh;
    const LcDev& ix = a.ix;
    const int b = blockIdx.y, tid = threadIdx.x, M = min(ix.state[b * ix.H * 4 + 1], ix.cap[0]);
    const int* bnd = ix.bounds + (size_t)b * (ix.cap[0] + 1);
    int32_t* spare = a.spare + (size_t)b * 2 * ix.cap[0];
    const int last = bnd[M];
    int tok = 0;
    uint32_t lo = 0xffffffffu, hi = 0u;
    lc_evict_range(a, b, lo, hi, tok);
    lc_cut_prepare(sh);
    lo = (uint32_t)lc_readlane((int)lc_wave_extreme<false>(lo), 63);
    hi = (uint32_t)lc_readlane((int)lc_wave_extreme<true>(hi), 63);
    const int others = lc_readlane(lc_wave_scan_incl(tok), 63), left = max(0, a.keep - (last - others));
    if (others <= left) {                                    // (all stay)
        if (blockIdx.x == 0 && tid == 0) spare[LC_EVS_CUT + 3] = -1;
        return;
    }
    LcCut cut = lc_cut_of(lo, hi, left);
    __syncthreads();
    lc_slab_each(LcSlab(M, blockIdx.x, gridDim.x), bnd, a.keys + (size_t)b * ix.cap[0], [&](int, int n, unsigned long long k, bool real) LC_INLINE {
        int d;
        if (cut.digit(k, &d) && real) atomicAdd(&sh.tok[d], n);
    });
    __syncthreads();
    for (int i = tid; i < LC_EV_BINS; i += LC_EV_THREADS)
        if (sh.tok[i] != 0) __hip_atomic_fetch_add(spare + i, sh.tok[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (!lc_arrive_last(&ix.sync[b * ix.H * 4 + 2], gridDim.x, &sh.few)) return;
    const uint32_t* digits = reinterpret_cast<const uint32_t*>(spare);
    const int d1 = LC_EV_BINS - 1 - 2 * tid, t1 = (int)lc_load_agent(digits + d1), t0 = (int)lc_load_agent(digits + d1 - 1);
    lc_cut_digit(sh, cut, t1, t0, false);
    if (tid == 0) {
        spare[LC_EVS_CUT] = (int32_t)(uint32_t)cut.base;
        spare[LC_EVS_CUT + 1] = (int32_t)(uint32_t)(cut.base >> 32);
        spare[LC_EVS_CUT + 2] = cut.shift;
        spare[LC_EVS_CUT + 3] = cut.left;
        ix.sync[b * ix.H * 4 + 2] = 0;                       // ready for the next launch
    }
}

__global__ void __launch_bounds__(LC_EV_THREADS)
lc_evict_sift_kernel(const LcEvictArgs a) {
    lc_fetch_args<sizeof(LcEvictArgs)>();
    constexpr int NW = LC_EV_THREADS / 64;
    __shared__ LcCutSh sh;
    __shared__ int red_sh[2 * NW];
    const LcDev& ix = a.ix;
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, M = min(ix.state[b * ix.H * 4 + 1], ix.cap[0]);
    const int* bnd = ix.bounds + (size_t)b * (ix.cap[0] + 1);
    const unsigned long long* keys = a.keys + (size_t)b * ix.cap[0];
    int32_t* spare = a.spare + (size_t)b * 2 * ix.cap[0];
    int32_t* const list = spare + LC_EVS_RANGE + 3 * a.sums;
    const LcSlab slab(M, blockIdx.x, gridDim.x);
    const LcCut cut = {(unsigned long long)(uint32_t)spare[LC_EVS_CUT] | (unsigned long long)(uint32_t)spare[LC_EVS_CUT + 1] << 32, spare[LC_EVS_CUT + 2], spare[LC_EVS_CUT + 3]};
    lc_cut_prepare(sh);
    uint32_t* const mine = reinterpret_cast<uint32_t*>(spare + LC_EVS_KEPT + 2 * blockIdx.x);
    if (cut.left < 0) {                                      // (all stay)
        if (tid == 0) {
            mine[0] = (uint32_t)(slab.hi - slab.lo);
            mine[1] = (uint32_t)(bnd[slab.hi] - bnd[slab.lo]);
            if (blockIdx.x == 0) { spare[LC_EVS_LAST] = spare[LC_EVS_LAST + 1] = 0; spare[LC_EVS_LAST + 2] = 0x7fffffff; }
        }
        return;
    }
    int count = 0, tokens = 0;
    lc_slab_each(slab, bnd, keys, [&](int j, int n, unsigned long long k, bool real) LC_INLINE {
        const bool above = real && cut.above(k), at = real && cut.at(k);
        count += above ? 1 : 0;
        tokens += above ? n : 0;
        const unsigned long long m = __ballot(at);
        if (m != 0ull) {
            int place = 0;
            if (lane == 0) place = __hip_atomic_fetch_add(spare + LC_EVS_N, __popcll(m), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            place = lc_readlane(place, 0) + __popcll(m & ((1ull << lane) - 1ull));
            if (at) lc_store_agent(reinterpret_cast<uint32_t*>(list + place), (uint32_t)j);
        }
    });
    count = lc_wave_scan_incl(count);
    tokens = lc_wave_scan_incl(tokens);
    if (lane == 63) { red_sh[wave] = count; red_sh[NW + wave] = tokens; }
    __syncthreads();
    if (tid == 0) {
        count = tokens = 0;
        for (int w = 0; w < NW; ++w) { count += red_sh[w]; tokens += red_sh[NW + w]; }
        lc_store_agent(mine, (uint32_t)count);
        lc_store_agent(mine + 1, (uint32_t)tokens);
    }
    if (!lc_arrive_last(&ix.sync[b * ix.H * 4 + 2], gridDim.x, red_sh)) return;
    // the chunks at the cut: one in a thread's registers, the others, if there are so many, where they are
    const int listed = min((int)lc_load_agent(reinterpret_cast<const uint32_t*>(spare + LC_EVS_N)), M);
    auto entry = [&](int i, int* n, unsigned long long* k) LC_INLINE -> int {
        const int j = min((int)lc_load_agent(reinterpret_cast<const uint32_t*>(list + i)), M - 1);
        *n = bnd[j + 1] - bnd[j];
        *k = keys[j];
        return j;
    };
    int j1 = 0, n1 = 0;
    unsigned long long k1 = LC_EV_PINNED;
    if (tid < listed) j1 = entry(tid, &n1, &k1);
    auto each = [&](auto f) LC_INLINE {
        f(j1, n1, k1);
        for (int i = tid + LC_EV_THREADS; i < listed; i += LC_EV_THREADS) {
            int n;
            unsigned long long k;
            const int j = entry(i, &n, &k);
            f(j, n, k);
        }
    };
    lc_cut_search(sh, cut, true, M, each, [&](int j, int* n) LC_INLINE {
        *n = bnd[j + 1] - bnd[j];
        return keys[j];
    });
    const unsigned long long last_key = sh.last_key;
    const int last_id = sh.last_id;
    each([&](int j, int n, unsigned long long k) LC_INLINE {
        if (k != LC_EV_PINNED && (k > last_key || (k == last_key && j <= last_id))) {
            int32_t* const whose = spare + LC_EVS_KEPT + 2 * (j / slab.size);
            __hip_atomic_fetch_add(whose, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_fetch_add(whose + 1, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    });
    if (tid == 0) {
        spare[LC_EVS_LAST] = (int32_t)(uint32_t)last_key;
        spare[LC_EVS_LAST + 1] = (int32_t)(uint32_t)(last_key >> 32);
        spare[LC_EVS_LAST + 2] = last_id;
        ix.sync[b * ix.H * 4 + 2] = 0;                       // ready for the next launch
    }
}

__global__ void __launch_bounds__(LC_EV_THREADS)
lc_evict_place_kernel(const LcEvictArgs a) {
    lc_fetch_args<sizeof(LcEvictArgs)>();
    __shared__ int scan_sh[2 * (LC_EV_THREADS / 64)];
    const LcDev& ix = a.ix;
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, T = ix.state[b * ix.H * 4 + 0], M = min(ix.state[b * ix.H * 4 + 1], ix.cap[0]);
    const int* bnd = ix.bounds + (size_t)b * (ix.cap[0] + 1);
    const unsigned long long* keys = a.keys + (size_t)b * ix.cap[0];
    const int32_t* spare = a.spare + (size_t)b * 2 * ix.cap[0];
    const LcSlab slab(M, blockIdx.x, gridDim.x);
    const unsigned long long last_key = (unsigned long long)(uint32_t)spare[LC_EVS_LAST] | (unsigned long long)(uint32_t)spare[LC_EVS_LAST + 1] << 32;
    const int last_id = spare[LC_EVS_LAST + 2], last = bnd[M];
    // what the workgroups before this one keep, and all
    int n_keep = 0, n_tok = 0, all_keep = 0, all_tok = 0;
    for (int i = lane; i < (int)gridDim.x; i += 64) {
        const int c = spare[LC_EVS_KEPT + 2 * i], t = spare[LC_EVS_KEPT + 2 * i + 1];
        all_keep += c;
        all_tok += t;
        n_keep += i < (int)blockIdx.x ? c : 0;
        n_tok += i < (int)blockIdx.x ? t : 0;
    }
    auto sum = [&](int v) LC_INLINE { return lc_readlane(lc_wave_scan_incl(v), 63); };
    n_keep = sum(n_keep);
    n_tok = sum(n_tok);
    all_keep = sum(all_keep);
    all_tok = sum(all_tok);
    int32_t* ids = a.ids + (size_t)b * ix.cap[0];
    int32_t* bounds = a.bounds + (size_t)b * (ix.cap[0] + 1);
    lc_evict_place(slab.lo, slab.hi, bnd, ids, bounds, scan_sh, n_keep, n_tok, [&](int j, const int*) LC_INLINE {
        uint32_t kept = 0u;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const unsigned long long k = keys[min(j + u, slab.hi - 1)];
            kept |= j + u < slab.hi && (k > last_key || (k == last_key && j + u <= last_id)) ? 1u << u : 0u;
        }
        return kept;
    });
    for (int i = all_keep + (int)blockIdx.x * LC_EV_THREADS + tid; i < ix.cap[0]; i += (int)gridDim.x * LC_EV_THREADS) {
        ids[i] = -1;
        bounds[i] = all_tok;
    }
    if (blockIdx.x == 0 && tid == 0) {
        bounds[ix.cap[0]] = all_tok;
        a.counts[b] = all_keep;
        if (a.lens) a.lens[b] = all_tok + max(0, T - last);
    }
}

// ---------------------------------------------------------------- the rows that stay
#define LC_ER_THREADS 256
#define LC_ER_ROWS 64             // new rows of a tile
#define LC_ER_STREAM (32LL << 20)         // bytes of keys and values from which on bfloat16 rows go past the caches
#define LC_ER_GROUPS 32768        // workgroups for rows at most; each goes on to further tiles
#define LC_ER_WEIGHTS 64          // workgroups of a (sequence, head) for weights at most
#define LC_ER_GROUPS4 4096        // ... in 4 bits, where a tile is a few KB and those past the kept rows' end are not free (25 us without, 23 with)

struct LcEvictRowsArgs {
    LcDev ix;
    const int32_t *ids, *bounds, *counts;
    const char *K, *V;
    char *K_to, *V_to;
    long long seq, head, tok, seq_to, head_to, tok_to;    // strides in bytes
    const float* weights;
    float* weights_to;
    int max_tokens;
    int row_tiles;        // workgroups that move rows; those behind move weights
};

// The piece of a 4-bit row that a lane moves at a time: rows are 4-byte aligned.
typedef int LcPiece4 __attribute__((ext_vector_type(4), aligned(4)));

// A tile is ROWS new rows of a (sequence, head), keys and values: the rows of the kept chunks one behind the other, then the open tail's; a chain of five loads
// finds them.  Bound by the bytes where chunks are long: half of 32K tokens of 4 sequences, 8 heads, bfloat16, 538 MB, in 95 us (5.7 TB/s; through the caches 114,
// with 4096 workgroups that go on to further tiles instead of a tile each 102, with the heads of a tile one after the other 102), of one sequence 27 us (33 through the caches; half of 8K tokens, 34 MB: 9.7 either way,
// a quarter of 4K 4.9 through them, 6.0 past them).  Chunks of a dozen tokens in 4 bits are runs of 0.8 KB, which the memory reads at 3.1 TB/s of useful bytes: 128K
// tokens cut to a quarter 23 us.  (There tiles of 128 and 256 rows take 24.6 and 28.3; past the caches, where rows share lines, 32; several heads to a workgroup, which share
// the rows' places, 23.9 to 26.6.)
template <int BYTES, int ROWS, bool STREAM>    // bytes of a row; past the caches
__global__ void __launch_bounds__(LC_ER_THREADS)
lc_evict_rows_kernel(const LcEvictRowsArgs a) {
    lc_fetch_args<sizeof(LcEvictRowsArgs)>();
    __shared__ int bound_sh[ROWS], begin_sh[ROWS];
    __shared__ int row_sh[ROWS];
    const LcDev& ix = a.ix;
    const int h = blockIdx.y, b = blockIdx.z, bh = b * ix.H + h, part = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    const int cap = ix.cap[0];
    const int32_t* ids = a.ids + (size_t)b * cap;
    const int32_t* kept = a.bounds + (size_t)b * (cap + 1);
    const int T = min(ix.state[bh * 4 + 0], a.max_tokens), M = min(ix.state[bh * 4 + 1], cap);
    const int* bnd = ix.bounds + (size_t)b * (cap + 1);
    const int n = max(0, min(a.counts[b], M));
    if (part >= a.row_tiles) {
        for (int i = (part - a.row_tiles) * LC_ER_THREADS + tid; i < cap; i += ((int)gridDim.x - a.row_tiles) * LC_ER_THREADS) {
            const int id = i < n ? ids[i] : -1;
            a.weights_to[(size_t)bh * cap + i] = id >= 0 && id < M ? a.weights[(size_t)bh * cap + id] : 0.f;
        }
        return;
    }
    const int last = bnd[M], n_kept = max(0, min(kept[n], T)), rows = min(n_kept + max(0, T - last), a.max_tokens);
    const size_t from = (size_t)b * a.seq + (size_t)h * a.head, to = (size_t)b * a.seq_to + (size_t)h * a.head_to;
    for (int r0 = part * ROWS; r0 < rows; r0 += a.row_tiles * ROWS) {
        // the last kept chunk that begins at or before r0: 64 boundaries at a time, each round a 64th of the range
        int lo = 0, len = n;                                 // boundaries lo .. lo + len - 1 are candidates, kept[lo] <= r0
        while (len > 1) {
            const int step = (len + 63) / 64;
            const int i = lane * step;
            const bool below = i < len && kept[lo + i] <= r0;
            const unsigned long long m = __ballot(below);
            const int at = (63 - __clzll((long long)(m | 1ull))) * step;
            lo += at;
            len = min(step, len - at);
        }
        // a row lies in one of the next ROWS chunks, or behind them all in the tail
        if (tid < ROWS) {
            const bool real = lo + tid < n;
            const int at = real ? kept[lo + tid] : 0x7fffffff, id = real ? ids[lo + tid] : 0;
            bound_sh[tid] = at;
            begin_sh[tid] = bnd[max(0, min(id, M - 1))];
        }
        __syncthreads();
        if (tid < ROWS) {
            const int r = r0 + tid;
            int row = last + (r - n_kept);
            if (r < n_kept) {
                int i = 0;
#pragma unroll
                for (int s = ROWS / 2; s > 0; s >>= 1)
                    if (bound_sh[i + s] <= r) i += s;
                row = begin_sh[i] + (r - bound_sh[i]);
            }
            row_sh[tid] = max(0, min(row, T - 1));
        }
        __syncthreads();
        const int m = min(ROWS, rows - r0);
        // (all of a thread's loads before its stores)
        using Piece = typename std::conditional<BYTES % 16 == 0, lc_v4i, LcPiece4>::type;
        constexpr int PIECES = BYTES / 16, PER = ROWS * PIECES / LC_ER_THREADS;
        static_assert(BYTES - 16 * PIECES == 0 || (BYTES - 16 * PIECES == 4 && ROWS <= LC_ER_THREADS), "");
        lc_v4i k[PER], v[PER];
        uint32_t ks = 0u, vs = 0u;
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int i = tid + u * LC_ER_THREADS, r = i / PIECES;
            if (r < m) {
                const size_t f = from + (size_t)row_sh[r] * a.tok + i % PIECES * 16;
                if constexpr (STREAM) {
                    k[u] = __builtin_nontemporal_load(reinterpret_cast<const Piece*>(a.K + f));
                    v[u] = __builtin_nontemporal_load(reinterpret_cast<const Piece*>(a.V + f));
                } else {
                    k[u] = *reinterpret_cast<const Piece*>(a.K + f);
                    v[u] = *reinterpret_cast<const Piece*>(a.V + f);
                }
            }
        }
        if (BYTES % 16 != 0 && tid < m) {
            const size_t f = from + (size_t)row_sh[tid] * a.tok + 16 * PIECES;
            ks = *reinterpret_cast<const uint32_t*>(a.K + f);
            vs = *reinterpret_cast<const uint32_t*>(a.V + f);
        }
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int i = tid + u * LC_ER_THREADS, r = i / PIECES;
            if (r < m) {
                const size_t t = to + (size_t)(r0 + r) * a.tok_to + i % PIECES * 16;
                if constexpr (STREAM) {
                    __builtin_nontemporal_store((Piece)k[u], reinterpret_cast<Piece*>(a.K_to + t));
                    __builtin_nontemporal_store((Piece)v[u], reinterpret_cast<Piece*>(a.V_to + t));
                } else {
                    *reinterpret_cast<Piece*>(a.K_to + t) = k[u];
                    *reinterpret_cast<Piece*>(a.V_to + t) = v[u];
                }
            }
        }
        if (BYTES % 16 != 0 && tid < m) {
            const size_t t = to + (size_t)(r0 + tid) * a.tok_to + 16 * PIECES;
            *reinterpret_cast<uint32_t*>(a.K_to + t) = ks;
            *reinterpret_cast<uint32_t*>(a.V_to + t) = vs;
        }
        __syncthreads();                                     // (the lists have been used)
    }
}

// ---------------------------------------------------------------- arguments
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int check_strides16(const int64_t s[3]) {
    if (!s) return LC_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || s[i] % 8 != 0) return LC_ERR_BAD_SHAPE;
    return s[2] < LC_HEAD_DIM ? LC_ERR_BAD_SHAPE : LC_OK;
}

int weigh(const lc_index* idx, const void* q, const void* K, const int64_t s[3], bool in4, const int32_t* chunk_ids, const int32_t* counts, int cap,
          int H_q, const float* lse, float* weights, void* stream) {
    if (!idx || !q) return LC_ERR_INVALID_ARG;
    if (H_q < idx->H_kv || H_q % idx->H_kv != 0 || H_q / idx->H_kv > LC_MAX_GROUP) return LC_ERR_BAD_SHAPE;
    if (cap < 1 || !K || !chunk_ids || !counts || !lse || !weights) return LC_ERR_INVALID_ARG;
    const int rc = in4 ? lc_check_strides4(s) : check_strides16(s);
    if (rc) return rc;
    if (!aligned(q, 16) || !aligned(K, in4 ? 4 : 16)) return LC_ERR_INVALID_ARG;
    const int cell = in4 ? 1 : 2;
    if ((long long)idx->cfg.max_tokens * s[2] * cell >= (1LL << 31) - 512) return LC_ERR_BAD_SHAPE;
    LcWeighArgs a;
    a.ix = idx->dev;
    a.q = static_cast<const uint16_t*>(q);
    a.K = K;
    a.seq = s[0] * cell; a.head = s[1] * cell; a.tok = (int)(s[2] * cell);
    a.max_tokens = idx->cfg.max_tokens;
    a.ids = chunk_ids;
    a.counts = counts;
    a.cap = cap;
    a.lse = lse;
    a.weights = weights;
    a.G = H_q / idx->H_kv;
    return in4 ? launch_weigh<true>(a, static_cast<hipStream_t>(stream)) : launch_weigh<false>(a, static_cast<hipStream_t>(stream));
}

int evict_rows(const lc_index* idx, const int32_t* keep_ids, const int32_t* keep_bounds, const int32_t* keep_counts, const void* K, const void* V,
               const int64_t s[3], void* K_to, void* V_to, const int64_t s_to[3], bool in4, const float* weights, float* weights_to, void* stream) {
    if (!idx || !keep_ids || !keep_bounds || !keep_counts || !K || !V || !K_to || !V_to) return LC_ERR_INVALID_ARG;
    if ((weights != nullptr) != (weights_to != nullptr)) return LC_ERR_INVALID_ARG;
    int rc = in4 ? lc_check_strides4(s) : check_strides16(s);
    if (rc == LC_OK) rc = in4 ? lc_check_strides4(s_to) : check_strides16(s_to);
    if (rc) return rc;
    const uintptr_t al = in4 ? 4 : 16;
    if (!aligned(K, al) || !aligned(V, al) || !aligned(K_to, al) || !aligned(V_to, al)) return LC_ERR_INVALID_ARG;
    if (K == K_to || V == V_to || K == V_to || V == K_to || K_to == V_to || (weights && weights == weights_to)) return LC_ERR_INVALID_ARG;
    const int cell = in4 ? 1 : 2;
    LcEvictRowsArgs a;
    a.ix = idx->dev;
    a.ids = keep_ids; a.bounds = keep_bounds; a.counts = keep_counts;
    a.K = static_cast<const char*>(K); a.V = static_cast<const char*>(V);
    a.K_to = static_cast<char*>(K_to); a.V_to = static_cast<char*>(V_to);
    a.seq = s[0] * cell; a.head = s[1] * cell; a.tok = s[2] * cell;
    a.seq_to = s_to[0] * cell; a.head_to = s_to[1] * cell; a.tok_to = s_to[2] * cell;
    a.weights = weights; a.weights_to = weights_to;
    a.max_tokens = idx->cfg.max_tokens;
    int most = 0;
    for (int b = 0; b < idx->B; ++b)
        if (idx->T[b] > most) most = idx->T[b];
    const int tiles = most > LC_ER_ROWS ? (most + LC_ER_ROWS - 1) / LC_ER_ROWS : 1, fit = ((in4 ? LC_ER_GROUPS4 : LC_ER_GROUPS) + idx->B * idx->H_kv - 1) / (idx->B * idx->H_kv);
    a.row_tiles = tiles < fit ? tiles : fit;
    const int slots = (idx->cfg.max_chunks + LC_ER_THREADS - 1) / LC_ER_THREADS, weight_tiles = weights ? (slots < LC_ER_WEIGHTS ? slots : LC_ER_WEIGHTS) : 0;
    const dim3 grid(a.row_tiles + weight_tiles, idx->H_kv, idx->B);
    hipStream_t st = static_cast<hipStream_t>(stream);
    long long rows = 0;
    for (int b = 0; b < idx->B; ++b) rows += idx->T[b];
    const dim3 block(LC_ER_THREADS);
    if (in4) hipLaunchKernelGGL((lc_evict_rows_kernel<LC_ROW4, LC_ER_ROWS, false>), grid, block, 0, st, a);
    else if (rows * idx->H_kv * (4 * LC_D) > LC_ER_STREAM) hipLaunchKernelGGL((lc_evict_rows_kernel<2 * LC_D, LC_ER_ROWS, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((lc_evict_rows_kernel<2 * LC_D, LC_ER_ROWS, false>), grid, block, 0, st, a);
    LC_HIP_CHECK(hipGetLastError());
    return LC_OK;
}

}  // namespace

extern "C" {

int lc_weigh_chunks(const lc_index* idx, const void* q, const void* K, const int64_t k_strides[3], const int32_t* chunk_ids, const int32_t* counts,
                    int cap, int H_q, const float* lse, float* weights, void* stream) {
    return weigh(idx, q, K, k_strides, false, chunk_ids, counts, cap, H_q, lse, weights, stream);
}

int lc_weigh_chunks4(const lc_index* idx, const void* q, const void* K4, const int64_t strides4[3], const int32_t* chunk_ids, const int32_t* counts,
                     int cap, int H_q, const float* lse, float* weights, void* stream) {
    return weigh(idx, q, K4, strides4, true, chunk_ids, counts, cap, H_q, lse, weights, stream);
}

int lc_evict_select(const lc_index* idx, const float* weights, int keep_tokens, int recent_tokens, int32_t* keep_ids, int32_t* keep_bounds,
                    int32_t* keep_counts, int32_t* keep_lens, void* ws, size_t ws_bytes, void* stream) {
    if (!idx || !weights || !keep_ids || !keep_bounds || !keep_counts || !ws || !aligned(ws, 256)) return LC_ERR_INVALID_ARG;
    if (keep_tokens < 0 || recent_tokens < 0) return LC_ERR_INVALID_ARG;
    const size_t keys_bytes = (size_t)idx->B * idx->cfg.max_chunks * sizeof(unsigned long long);
    if (ws_bytes < (idx->cfg.max_chunks > LC_EV_SINGLE_MAX ? 2 * keys_bytes : keys_bytes)) return LC_ERR_WORKSPACE_TOO_SMALL;
    unsigned long long* keys = static_cast<unsigned long long*>(ws);
    hipStream_t st = static_cast<hipStream_t>(stream);
    int most = 0;
    for (int b = 0; b < idx->B; ++b)
        if (idx->M[b] > most) most = idx->M[b];
    LcEvictArgs a;
    a.ix = idx->dev;
    a.weights = weights;
    a.keys = keys;
    a.ids = keep_ids; a.bounds = keep_bounds; a.counts = keep_counts; a.lens = keep_lens;
    a.keep = keep_tokens; a.recent = recent_tokens; a.sink = idx->cfg.sink_tokens;
    a.sums = (most + LC_EV_SUM - 1) / LC_EV_SUM;
    a.range = keep_ids;                                      // (room for more than that, and written behind all else)
    a.range_seq = idx->cfg.max_chunks;
    a.spare = nullptr;
    const dim3 grid(idx->B), block(LC_EV_THREADS);
    if (most <= LC_EV_FUSED_MAX) {
        if (most <= LC_EV_THREADS) hipLaunchKernelGGL((lc_evict_select_kernel<1, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((lc_evict_select_kernel<4, true>), grid, block, 0, st, a);
    } else if (most <= LC_EV_SINGLE_MAX) {
        hipLaunchKernelGGL(lc_evict_keys_kernel, dim3(a.sums, idx->B), dim3(LC_EV_SUM), 0, st, a);
        LC_HIP_CHECK(hipGetLastError());
        hipLaunchKernelGGL((lc_evict_select_kernel<12, false>), grid, block, 0, st, a);
    } else {
        a.spare = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + keys_bytes);
        a.range = a.spare + LC_EVS_RANGE;
        a.range_seq = 2 * (long long)idx->cfg.max_chunks;
        const int slabs = (most + LC_EV_SLAB - 1) / LC_EV_SLAB;
        const dim3 shared(slabs < LC_EV_GROUPS ? slabs : LC_EV_GROUPS, idx->B);
        hipLaunchKernelGGL(lc_evict_keys_kernel, dim3(a.sums, idx->B), dim3(LC_EV_SUM), 0, st, a);
        LC_HIP_CHECK(hipGetLastError());
        hipLaunchKernelGGL(lc_evict_cut_kernel, shared, block, 0, st, a);
        LC_HIP_CHECK(hipGetLastError());
        hipLaunchKernelGGL(lc_evict_sift_kernel, shared, block, 0, st, a);
        LC_HIP_CHECK(hipGetLastError());
        hipLaunchKernelGGL(lc_evict_place_kernel, shared, block, 0, st, a);
    }
    LC_HIP_CHECK(hipGetLastError());
    return LC_OK;
}

int lc_evict_rows(const lc_index* idx, const int32_t* keep_ids, const int32_t* keep_bounds, const int32_t* keep_counts, const void* K, const void* V,
                  const int64_t kv_strides[3], void* K_to, void* V_to, const int64_t to_strides[3], const float* weights, float* weights_to, void* stream) {
    return evict_rows(idx, keep_ids, keep_bounds, keep_counts, K, V, kv_strides, K_to, V_to, to_strides, false, weights, weights_to, stream);
}

int lc_evict_rows4(const lc_index* idx, const int32_t* keep_ids, const int32_t* keep_bounds, const int32_t* keep_counts, const void* K4, const void* V4,
                   const int64_t strides4[3], void* K4_to, void* V4_to, const int64_t to_strides4[3], const float* weights, float* weights_to, void* stream) {
    return evict_rows(idx, keep_ids, keep_bounds, keep_counts, K4, V4, strides4, K4_to, V4_to, to_strides4, true, weights, weights_to, stream);
}

}  // extern "C"
