// A cache of keys and values in 4 bits: rows stored and loaded (lc_cache4_store, lc_cache4_load), and the sparse attention
// of one decode step over it (lc_sparse_decode4).  The row format is lc_cache4.h's.
//
// Attention.  With x_t = q.k_t / sqrt(d) over the tokens of the listed chunks and of the open tail,
//   out = sum_t e^(x_t - m) v_t / sum_t e^(x_t - m),   lse = m + ln sum_t e^(x_t - m),
// in one pass over the rows: each wavefront keeps a reference m of its own (a whole number of powers of two, not below its largest logit so far), the
// parts meet at the end.  Grid (KV head, sequence, split), 256 threads; a wavefront takes 32 tokens at a time.
//   Q.K^T: the 16 tokens of half a step are the rows of a 16x16x32 bf16 product's A operand, lane (kg, n) holding the 32 columns [32 kg, ...) of
//   row n -- one 16-byte load, whose scale is one byte -- as four operands of eight; the query block is the B operand.  The products leave lane
//   (kg, n) the logits of tokens 4 kg .. 4 kg + 3 for the head of column n.
//   P.V: a lane's eight probabilities (of the two halves) are its share of the B operand, and the eight columns [8 n, 8 n + 8) of the same eight
//   tokens -- one 4-byte load each -- are, column by column, its share of eight A operands.  No value crosses lanes.  A probability goes in as three bfloat16 terms
//   that add up to its float32 value; the terms of a head stand in columns of their own, whose logits are the head's once more, so that up to
//   group size 5 one product takes all three (the matrix pipe multiplies 16 columns whatever is in them); above, the third term takes a second one.
// Error against float64: 1.3e-7 to 2.1e-7 of the output's size over the sizes below.  (The 16x16x128 product on 4- and 8-bit operands with a scale
// per 32 would take the rows as they are, with the query in two e4m3 terms that hold it exactly: it adds up its products aligned to the largest of them,
// 4.5e-5 of the result's size off on random operands of that kind.)
//
// Measured (kernel alone, replayed from a graph, cold rows): 1024 of 4K tokens, 8 heads of group size 4, 8.2 us; 4096 of 128K tokens 9.7
// (with the long lists' code between the other in the kernel 0.1 more, with all 16 reads of a merging thread however few splits there are another 0.3); 16 ragged sequences, 4
// heads of group size 7, 2048 tokens each 13.9; all of 4 x 128K tokens 119 (570 MB: 4.8 TB/s, one behind the other 5.2).  lc_sparse_decode over bfloat16 rows: 8.2, 10.9, 19.1 and 390.
// Long lists are bound by the bytes: without arithmetic the last one takes 4 us less, with all rows from the caches 96.  Short ones are a chain: launch 1.4, the list 0.7,
// boundaries and their sums 0.6, rows' places 1.4, rows 0.5, a step 0.9, sums through LDS and out 1.1, arrival 0.5, merge 1.2.
// Other ways: three steps on their way instead of two 130.7 us (129 with two at that stage); three or four workgroups per compute unit spill registers; rows past
// the caches 154 (lines that several loads share come twice); the list held by every wavefront, without barriers, 10.0 and 121; rows found by each wavefront
// for its own steps from marks that the entries leave at their first tokens, one barrier instead of three, 8.5 and 122.
#include "lc_cache4.h"
#include "lc_internal.h"
#include "lc_select.h"

#define LC_C4_THREADS 256
#define LC_C4_ROWS 64             // rows that a workgroup stores or loads
#define LC_C4_BATCH 64            // sequences of a launch: their row numbers are launch arguments
#define LC_D4_THREADS 256
#define LC_D4_WAVES (LC_D4_THREADS / 64)
#define LC_D4_TILE 8192           // tokens of a split whose cache rows are resolved into LDS at a time (all of 4 x 128K tokens: 135 us, with 1024 146, at that stage)
#define LC_D4_MIN_TOKENS 128      // tokens of a split, at least: a step of each wavefront (8 heads of 1024 tokens: 8.7 us, with 64 9.0, with 256 9.4; of 2048: 8.9, 9.7, 9.5)
#define LC_D4_E 8                 // listed chunks per thread and pass of the row resolution
#define LC_D4_MAX_SPLITS 256
#define LC_LOG2E 1.4426950408889634f
#define LC_LN2 0.6931471805599453f
#define LC_INLINE __attribute__((always_inline))

namespace {

// ---------------------------------------------------------------- rows
struct LcRange4 { int32_t first[LC_C4_BATCH], count[LC_C4_BATCH]; };

struct LcMove4Args {
    uint16_t *K, *V;
    uint8_t *K4, *V4;
    long long seq, head, tok;         // strides of K and V, in values
    long long seq4, head4, tok4;      // strides of K4 and V4, in bytes
    LcRange4 r;
};

// Row i of the sequence's range: from row i of K or V to row first + i of K4 or V4.  16 lanes to a row, 64 rows to a workgroup; z: keys and values of
// each sequence in turn.  Bound by the bytes: 128K tokens of 8 heads, 680 MB, are stored in 116 us and loaded in 115 (5.9 TB/s).  The bfloat16 side, which nobody
// reads again soon, goes past the caches: 64K tokens are stored in 54 us (60 through them) and loaded in 50 (63).  Writing 16 bytes a lane, by way of
// LDS, was no faster than four; with the heads of a tile one after the other instead of the tiles of a head 128K tokens took 124 and 127.
__global__ void __launch_bounds__(LC_C4_THREADS)
lc_store4_kernel(const LcMove4Args a) {
    const int b = blockIdx.z >> 1, h = blockIdx.y, sub = threadIdx.x & 15, grp = threadIdx.x >> 4;
    const int n = a.r.count[b];
    const int r0 = blockIdx.x * LC_C4_ROWS + grp;
    if (blockIdx.x * LC_C4_ROWS >= n) return;
    const uint16_t* src = ((blockIdx.z & 1) ? a.V : a.K) + b * a.seq + h * a.head + 8 * sub;
    uint8_t* dst = ((blockIdx.z & 1) ? a.V4 : a.K4) + b * a.seq4 + h * a.head4 + (long long)a.r.first[b] * a.tok4;
    lc_v4i v[LC_C4_ROWS / 16];
#pragma unroll
    for (int k = 0; k < LC_C4_ROWS / 16; ++k) {
        const int r = r0 + 16 * k;
        v[k] = lc_v4i{0, 0, 0, 0};
        if (r < n) v[k] = __builtin_nontemporal_load(reinterpret_cast<const lc_v4i*>(src + r * a.tok));
    }
#pragma unroll
    for (int k = 0; k < LC_C4_ROWS / 16; ++k) {
        const int r = r0 + 16 * k;
        uint32_t scale;
        const uint32_t codes = lc_pack4(__builtin_bit_cast(uint4, v[k]), &scale);
        if (r < n) {
            uint8_t* row = dst + r * a.tok4;
            *reinterpret_cast<uint32_t*>(row + 4 * sub) = codes;
            if ((sub & 3) == 0) row[64 + (sub >> 2)] = (uint8_t)scale;
        }
    }
}

// Row first + i of K4 or V4 to row i of K or V.
__global__ void __launch_bounds__(LC_C4_THREADS)
lc_load4_kernel(const LcMove4Args a) {
    const int b = blockIdx.z >> 1, h = blockIdx.y, sub = threadIdx.x & 15, grp = threadIdx.x >> 4;
    const int n = a.r.count[b];
    const int r0 = blockIdx.x * LC_C4_ROWS + grp;
    if (blockIdx.x * LC_C4_ROWS >= n) return;
    uint16_t* dst = ((blockIdx.z & 1) ? a.V : a.K) + b * a.seq + h * a.head + 8 * sub;
    const uint8_t* src = ((blockIdx.z & 1) ? a.V4 : a.K4) + b * a.seq4 + h * a.head4 + (long long)a.r.first[b] * a.tok4;
    uint32_t c[LC_C4_ROWS / 16], s[LC_C4_ROWS / 16];
#pragma unroll
    for (int k = 0; k < LC_C4_ROWS / 16; ++k) {
        const int r = r0 + 16 * k;
        c[k] = s[k] = 0u;
        if (r < n) {
            c[k] = *reinterpret_cast<const uint32_t*>(src + r * a.tok4 + 4 * sub);
            s[k] = src[r * a.tok4 + 64 + (sub >> 2)];
        }
    }
#pragma unroll
    for (int k = 0; k < LC_C4_ROWS / 16; ++k) {
        const int r = r0 + 16 * k;
        if (r < n) __builtin_nontemporal_store(__builtin_bit_cast(lc_v4i, lc_unpack4(c[k], lc_scale4(s[k]))), reinterpret_cast<lc_v4i*>(dst + r * a.tok));
    }
}

// ---------------------------------------------------------------- attention
struct LcDecode4Args {
    LcDev ix;
    const uint16_t* q;
    const uint8_t *K, *V;
    long long seq, head;  // strides in bytes
    int tok;
    int max_tokens;       // rows of one (sequence, head) slab of K and V
    const int32_t* ids;
    const int32_t* counts;
    int cap;
    float* part_acc;      // [B][H][S][G][d]
    float* part_ml;       // [B][H][S][G][2]
    float* out;           // [B][H*G][d]
    float* lse;           // [B][H*G] or null
};

template <int G>
__global__ void __launch_bounds__(LC_D4_THREADS, 2)
lc_decode4_kernel(const LcDecode4Args a) {
    lc_fetch_args<sizeof(LcDecode4Args)>();
    constexpr bool WIDE = G > 5;                 // three terms of a probability in three columns, or two in two and the third apart
    constexpr int COLS = WIDE ? 16 : 3 * G;      // columns that hold something
    constexpr int TERMS = WIDE ? 2 : 3;          // columns of a head
    constexpr int STEP = 32;
    constexpr int E = LC_D4_E, PASS = E * LC_D4_THREADS;
    constexpr int ROW = LC_D + 4;                // floats between the columns' sums in LDS: lanes of different columns use different banks
    union Phases {
        struct {
            float acc[LC_D4_WAVES][COLS][ROW];
            float ml[LC_D4_WAVES][G][2];
        } comb;
        struct {
            float scale[LC_D4_THREADS / 32][LC_D4_MAX_SPLITS + 128], sum[LC_D4_THREADS / 32][LC_D4_MAX_SPLITS];
            float4 red[LC_D4_THREADS];
        } merge;
        int row[LC_D4_TILE + 2 * LC_D4_WAVES * STEP];    // byte offsets of the cache rows of the tile's tokens
    };
    __shared__ __attribute__((aligned(16))) Phases ph;
    __shared__ __attribute__((aligned(16))) int off_sh[E * LC_D4_THREADS + 4], st_sh[E * LC_D4_THREADS];
    __shared__ int scan_sh[8], slot_sh[64];
    __shared__ int first_sh, last_sh;

    const LcDev& ix = a.ix;
    const int s = blockIdx.z, S = gridDim.z, h = blockIdx.x, b = blockIdx.y;
    const int bh = b * ix.H + h;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, kg = lane >> 4;
    // the head and the term of this lane's column
    const int term = WIDE ? n >> 3 : n / G;
    const int head = WIDE ? min(n & 7, G - 1) : n - term * G;
    // which of a probability's terms come before this column's, as masks; and whether it has one (the third, where that is apart)
    const uint32_t past0 = term >= 1 ? 0xffff0000u : 0u, past1 = term >= 2 ? 0xffff0000u : 0u;
    const uint32_t here = WIDE ? (term == 0 ? 0xffffffffu : 0u) : (term < 3 ? 0xffffffffu : 0u);

    const __amdgpu_buffer_rsrc_t bnd_r = lc_buffer(ix.bounds + (size_t)b * (ix.cap[0] + 1), (ix.cap[0] + 1) * 4);
    const __amdgpu_buffer_rsrc_t ids_r = lc_buffer(a.ids + (size_t)bh * a.cap, (int)(min((long long)a.cap, 1LL << 28) * 4));

    // ---- the attended tokens: the listed chunks in the list's order, then the open tail.  Thread t of a pass owns entries [E t, E t + E);
    // the first pass stays in registers.
    struct Ids { lc_v4i v[E / 4]; };
    auto load_ids = [&](int base) LC_INLINE -> Ids {
        Ids w;
#pragma unroll
        for (int e = 0; e < E / 4; ++e) w.v[e] = __builtin_amdgcn_raw_buffer_load_b128(ids_r, (base + tid * E) * 4, 16 * e, 0);
        return w;
    };
    const Ids ids0 = load_ids(0);
    uint4 qb[4];
    {
        const uint16_t* qh = a.q + ((size_t)b * ix.H * G + (size_t)h * G + head) * LC_D + 32 * kg;
#pragma unroll
        for (int c = 0; c < 4; ++c) qb[c] = *reinterpret_cast<const uint4*>(qh + 8 * c);
    }
    const int T = ix.state[bh * 4 + 0], M = ix.state[bh * 4 + 1];
    const int n_ids = max(0, min(a.counts[bh], min(a.cap, 1 << 28)));
    const int tail_st = lc_buf_load_i32(bnd_r, M), tail_ln = max(0, T - tail_st);
    // (an entry that is no chunk holds no tokens)
    auto entries = [&](const Ids& ids, int base, int (&st)[E], int (&ln)[E]) LC_INLINE -> int {
        int sum = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int id = ids.v[e / 4][e % 4];
            const bool real = base + tid * E + e < n_ids && id >= 0 && id < M;
            // (branch-free: a load past the resource's end gives zeros)
            const lc_v2i x = __builtin_amdgcn_raw_buffer_load_b64(bnd_r, real ? id * 4 : 0x7ffffff0, 0, 0);
            st[e] = x.x;
            ln[e] = x.y;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            ln[e] = max(0, ln[e] - st[e]);
            sum += ln[e];
        }
        return sum;
    };
    int st0[E], ln0[E], tot0;
    if (tid < 64) slot_sh[tid] = 0;
    const int ex0 = lc_block_scan<LC_D4_THREADS>(entries(ids0, 0, st0, ln0), scan_sh, &tot0);
    // A longer list: the tokens of each of up to 64 slots of passes, so that a tile's rows are looked for in its own passes alone.
    const bool long_list = n_ids > PASS;
    const int passes = (n_ids + PASS - 1) / PASS, per_slot = (passes + 63) / 64;
    int n_sel = tot0, slot_end = 0;                          // (lane l: tokens up to the end of slot l)
    if (__builtin_expect(long_list, 0)) {
        Ids next = load_ids(PASS);
        for (int p = 1; p < passes; ++p) {
            const Ids now = next;
            if (p + 1 < passes) next = load_ids((p + 1) * PASS);
            int st[E], ln[E];
            const int sum = lc_wave_scan_incl(entries(now, p * PASS, st, ln));
            if (lane == 63) atomicAdd(&slot_sh[p / per_slot], sum);
        }
        if (tid == 0) atomicAdd(&slot_sh[0], tot0);
        __syncthreads();
        slot_end = lc_wave_scan_incl(slot_sh[lane]);
        n_sel = lc_readlane(slot_end, 63);
    }
    const int n_tok = n_sel + tail_ln;
    const int S_eff = max(1, min(S, (n_tok + LC_D4_MIN_TOKENS - 1) / LC_D4_MIN_TOKENS));
    if (s >= S_eff) return;                      // (the same n_tok in all of them: nobody waits for these)

    const float scale = 0.08838834764831845f * LC_LOG2E;     // log2(e) / sqrt(128)
    // The softmax of column n's head over the wavefront's tokens; acc[c][r]: column 8 (4 kg + r) + c of the values.
    float m_ref = LC_NEG_INF, l_run = 0.f;
    lc_f32x4 acc[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[c] = lc_f32x4{0.f, 0.f, 0.f, 0.f};
    // (the resources end with the last row the index may ever hold: past it, where tokens that are not there are read, loads give zeros)
    const int slab_bytes = (a.max_tokens - 1) * a.tok + LC_ROW4;
    const __amdgpu_buffer_rsrc_t Kr = lc_buffer(a.K + (size_t)b * a.seq + (size_t)h * a.head, slab_bytes);
    const __amdgpu_buffer_rsrc_t Vr = lc_buffer(a.V + (size_t)b * a.seq + (size_t)h * a.head, slab_bytes);

    struct Step {
        lc_v4i k[2];
        int ks[2];
        int v[8], vs[8];
    };
    auto load = [&](Step& w, int i) LC_INLINE {
        int ko[2], vo[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) ko[t] = ph.row[i + 16 * t + n];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const lc_v4i r = *reinterpret_cast<const lc_v4i*>(&ph.row[i + 16 * t + 4 * kg]);
#pragma unroll
            for (int j = 0; j < 4; ++j) vo[4 * t + j] = r[j];
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            w.k[t] = __builtin_amdgcn_raw_buffer_load_b128(Kr, ko[t] + 16 * kg, 0, 0);
            w.ks[t] = lc_buf_load_u8(Kr, ko[t] + 64 + kg);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) w.v[j] = __builtin_amdgcn_raw_buffer_load_b32(Vr, vo[j] + 4 * n, 0, 0);
#pragma unroll
        for (int j = 0; j < 8; ++j) w.vs[j] = lc_buf_load_u8(Vr, vo[j] + 64 + (n >> 2));
    };
    auto attend = [&](const Step& w, int i, int end) LC_INLINE {
        float x[8];
        float mx = LC_NEG_INF;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            lc_f32x4 d = {0.f, 0.f, 0.f, 0.f};
            const float f = lc_scale4((uint32_t)w.ks[t]);
#pragma unroll
            for (int c = 0; c < 4; ++c)
                d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(lc_bf16x8, lc_unpack4((uint32_t)w.k[t][c], f)),
                                                            __builtin_bit_cast(lc_bf16x8, qb[c]), d, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[4 * t + r] = i + 16 * t + 4 * kg + r < end ? d[r] : LC_NEG_INF;
                mx = fmaxf(mx, x[4 * t + r]);
            }
        }
        mx = lc_max_groups(mx) * scale;
        // (a whole number: scaling the sums by the difference of two rounds nothing)
        if (__ballot(mx > m_ref) != 0ull) {
            const float m_new = mx > m_ref ? ceilf(mx) : m_ref;
            const int by = m_ref == m_new ? 0 : (int)fmaxf(m_ref - m_new, -1024.f);
            m_ref = m_new;
            l_run = __builtin_ldexpf(l_run, by);
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[c][r] = __builtin_ldexpf(acc[c][r], by);
        }
        const float ref = m_ref == LC_NEG_INF ? 0.f : m_ref;
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_exp2f(fmaf(x[j], scale, -ref));
        l_run += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
        // the column's term of each probability: the upper eight bits of what the terms before have left
        lc_v4i t0, t1;
        {
            uint32_t w0[8], w1[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float r = p[j];
                r -= __uint_as_float(__float_as_uint(r) & past0);
                if constexpr (WIDE) {
                    const float r1 = p[j] - __uint_as_float(__float_as_uint(p[j]) & 0xffff0000u);
                    w0[j] = __float_as_uint(r);
                    w1[j] = __float_as_uint(r1 - __uint_as_float(__float_as_uint(r1) & 0xffff0000u)) & here;
                } else {
                    r -= __uint_as_float(__float_as_uint(r) & past1);
                    w0[j] = __float_as_uint(r) & here;
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                t0[j] = (int)__builtin_amdgcn_perm(w0[2 * j + 1], w0[2 * j], 0x07060302u);
                if constexpr (WIDE) t1[j] = (int)__builtin_amdgcn_perm(w1[2 * j + 1], w1[2 * j], 0x07060302u);
            }
        }
#pragma unroll
        for (int q2 = 0; q2 < 4; ++q2) {                        // columns 2 q2 and 2 q2 + 1 of this lane's eight
            uint32_t y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = lc_scale4((uint32_t)w.vs[j]);
                const uint32_t c = (uint32_t)w.v[j];
                y[j] = __builtin_bit_cast(uint32_t, q2 == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, f, 0)
                                                    : q2 == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, f, 1)
                                                    : q2 == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, f, 2)
                                                              : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, f, 3));
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                lc_v4i v;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = (int)__builtin_amdgcn_perm(y[2 * j + 1], y[2 * j], c ? 0x07060302u : 0x05040100u);
                lc_f32x4& o = acc[2 * q2 + c];
                if constexpr (WIDE)
                    o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(lc_bf16x8, v), __builtin_bit_cast(lc_bf16x8, t1), o, 0, 0, 0);
                o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(lc_bf16x8, v), __builtin_bit_cast(lc_bf16x8, t0), o, 0, 0, 0);
            }
        }
    };

    // ---- the split's tokens, in tiles whose rows the workgroup first writes into LDS
    const int each = (int)((uint32_t)n_tok / (uint32_t)S_eff), more = n_tok - each * S_eff;      // (the first `more` splits: one more)
    const int lo = each * s + min(s, more), hi = lo + each + (s < more ? 1 : 0);
    const int row_max = max(T - 1, 0);
    for (int tile0 = lo; tile0 < hi; tile0 += LC_D4_TILE) {
        const int tl = min(LC_D4_TILE, hi - tile0);
        // The entries' places in the list go into LDS, then 16 lanes take one entry that overlaps the tile, 16 tokens at a time.
        auto place = [&](int carry, int ex, int tot, int count, const int (&st)[E], const int (&ln)[E]) LC_INLINE {
            if (tile0 >= carry + tot || carry >= tile0 + tl) return;
            __syncthreads();                                        // (the entries before have been used)
            int off = carry + ex;
            if (tid == 0 && tile0 < carry) first_sh = 0;
            if (tid * E < count) {
                lc_v4i o[E / 4], f[E / 4];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    o[e / 4][e % 4] = off;
                    f[e / 4][e % 4] = st[e];
                    if (off <= tile0 && tile0 < off + ln[e]) first_sh = tid * E + e;
                    off += ln[e];
                }
#pragma unroll
                for (int e = 0; e < E / 4; ++e) {
                    reinterpret_cast<lc_v4i*>(off_sh)[tid * (E / 4) + e] = o[e];
                    reinterpret_cast<lc_v4i*>(st_sh)[tid * (E / 4) + e] = f[e];
                }
                if (tid * E + E >= count) off_sh[tid * E + E] = off;
            }
            __syncthreads();
            for (int i = first_sh + (tid >> 4); i < count; i += LC_D4_THREADS / 16) {
                const int o = off_sh[i], k1 = min(off_sh[i + 1], tile0 + tl), from = st_sh[i] - o;
                if (o >= tile0 + tl) break;
                for (int k = max(o, tile0) + n; k < k1; k += 16) ph.row[k - tile0] = min(from + k, row_max) * a.tok;
            }
        };
        if (tile0 != lo) __syncthreads();                           // the previous tile's rows have been used
        if (__builtin_expect(!long_list, 1)) {
            place(0, ex0, tot0, n_ids, st0, ln0);
        } else {
            const unsigned long long behind = __ballot(slot_end > tile0);
            const int slot = behind != 0ull ? __ffsll((long long)behind) - 1 : 64;
            int carry = slot == 64 ? n_sel : slot == 0 ? 0 : lc_readlane(slot_end, slot - 1);
            for (int p = slot * per_slot; p < passes && carry < tile0 + tl; ++p) {
                int st[E], ln[E], tot;
                const int ex = lc_block_scan<LC_D4_THREADS>(entries(load_ids(p * PASS), p * PASS, st, ln), scan_sh, &tot);
                place(carry, ex, tot, min(n_ids - p * PASS, PASS), st, ln);
                carry += tot;
            }
        }
        for (int k = max(n_sel, tile0) + tid; k < tile0 + tl; k += LC_D4_THREADS) ph.row[k - tile0] = min(tail_st + (k - n_sel), row_max) * a.tok;
        // Rounds of a step per wavefront; each fetches its rows while the round before is computed, without a branch around the loads (behind one the wait for
        // a step's rows would be for the next step's too), so that there are rows, past the resource's end, for up to two rounds more.
        const int rounds = (tl + LC_D4_WAVES * STEP - 1) / (LC_D4_WAVES * STEP);
        for (int k = tl + tid; k < (rounds + 2) * LC_D4_WAVES * STEP; k += LC_D4_THREADS) ph.row[k] = slab_bytes;
        __syncthreads();
        Step x, y;
        load(x, wave * STEP);
        for (int i = 0; i < rounds; i += 2) {
            const int at = (i * LC_D4_WAVES + wave) * STEP;
            load(y, at + LC_D4_WAVES * STEP);
            __builtin_amdgcn_sched_barrier(0);                      // (all of a round's loads are on their way before the round before is waited for)
            attend(x, at, tl);
            if (i + 1 >= rounds) break;
            load(x, at + 2 * LC_D4_WAVES * STEP);
            __builtin_amdgcn_sched_barrier(0);
            attend(y, at + LC_D4_WAVES * STEP, tl);
        }
    }

    // ---- the wavefronts' sums meet in LDS
    __syncthreads();
    {
        float l = lc_add_halves(l_run, l_run);
        l = lc_add_rows(l, l);
        if (kg == 0 && term == 0 && n < G) { ph.comb.ml[wave][head][0] = m_ref; ph.comb.ml[wave][head][1] = l; }
        if (n < COLS) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float4* const o = reinterpret_cast<float4*>(&ph.comb.acc[wave][n][8 * (4 * kg + r)]);
                o[0] = make_float4(acc[0][r], acc[1][r], acc[2][r], acc[3][r]);
                o[1] = make_float4(acc[4][r], acc[5][r], acc[6][r], acc[7][r]);
            }
        }
    }
    __syncthreads();
    auto finish = [&](int g, int c4, float4 num, float m, float den) LC_INLINE {
        const float inv = den == 0.f ? 0.f : 1.0f / den;           // (no tokens: zeros)
        const size_t o = (size_t)b * ix.H * G + (size_t)h * G + g;
        *reinterpret_cast<float4*>(a.out + o * LC_D + 4 * c4) = make_float4(num.x * inv, num.y * inv, num.z * inv, num.w * inv);
        if (a.lse && c4 == 0) {
            int e = 0;                                              // (whole powers of two aside, the logarithm is of a number near 1)
            const float part = den > 0.f ? frexpf(den, &e) : den;
            a.lse[o] = den == 0.f ? LC_NEG_INF : fmaf(m + (float)e, LC_LN2, logf(part));
        }
    };
    constexpr int NV = G * (LC_D / 4);                       // float4 slots of the output
    {
        float* pml = a.part_ml + ((size_t)bh * S + s) * G * 2;
        const __amdgpu_buffer_rsrc_t pacc_w = lc_buffer(a.part_acc + ((size_t)bh * S + s) * G * LC_D, G * LC_D * 4);
        for (int v = tid; v < NV; v += LC_D4_THREADS) {
            const int g = v / (LC_D / 4), c4 = v % (LC_D / 4);
            float m = LC_NEG_INF;
#pragma unroll
            for (int w = 0; w < LC_D4_WAVES; ++w) m = fmaxf(m, ph.comb.ml[w][g][0]);
            const float ref = m == LC_NEG_INF ? 0.f : m;
            float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
            float den = 0.f;
#pragma unroll
            for (int w = 0; w < LC_D4_WAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(ph.comb.ml[w][g][0] - ref);
#pragma unroll
                for (int t = TERMS - 1; t >= 0; --t) {
                    const float4 x = *reinterpret_cast<const float4*>(&ph.comb.acc[w][WIDE ? 8 * t + g : t * G + g][4 * c4]);
                    num.x = fmaf(x.x, f, num.x); num.y = fmaf(x.y, f, num.y);
                    num.z = fmaf(x.z, f, num.z); num.w = fmaf(x.w, f, num.w);
                }
                den = fmaf(ph.comb.ml[w][g][1], f, den);
            }
            if (S_eff == 1) {
                finish(g, c4, num, ref, den);
            } else {
                lc_store_agent4(pacc_w, v * 16, num);
                if (c4 == 0) { lc_store_agent(&pml[2 * g], m); lc_store_agent(&pml[2 * g + 1], den); }
            }
        }
    }
    if (S_eff == 1) return;

    // ---- the last split to arrive merges
    if (!lc_arrive_last(&ix.sync[bh * 4 + 1], S_eff, &last_sh)) return;
    const __amdgpu_buffer_rsrc_t pacc_r = lc_buffer(a.part_acc + (size_t)bh * S * G * LC_D, S_eff * G * LC_D * 4);
    const float* pml = a.part_ml + (size_t)bh * S * G * 2;
    constexpr int WAYS = (LC_D4_THREADS / NV) > 0 ? (LC_D4_THREADS / NV) : 1;
    constexpr int MR = 16;                                   // partials per round and thread
    const int v = tid % NV, wy = tid / NV;
    const int g = v / (LC_D / 4), c4 = v % (LC_D / 4);
    float4 x[MR];
    auto load_round = [&](int sp0) LC_INLINE {               // (by eights, as many as there are; past the last split: zeros)
#pragma unroll
        for (int k0 = 0; k0 < MR; k0 += 8)
            if (sp0 + k0 * WAYS < S_eff) {
#pragma unroll
                for (int k = k0; k < k0 + 8; ++k) x[k] = lc_load_agent4(pacc_r, (((sp0 + wy + k * WAYS) * G + g) * LC_D + 4 * c4) * 4);
            }
    };
    load_round(0);
    // Every 32 lanes have one head (slot v of the output) and turn its splits' references and sums into scales by themselves.
    const int half = tid >> 5, hl = tid & 31;
    float den = 0.f;
    float m0 = LC_NEG_INF, l0 = 0.f;                         // (the first 32 stay in registers)
    if (hl < S_eff) {
        m0 = lc_load_agent(pml + 2 * (hl * G + g));
        l0 = lc_load_agent(pml + 2 * (hl * G + g) + 1);
    }
    float m_all = m0;
    for (int sp = hl + 32; sp < S_eff; sp += 32) {
        const float m = lc_load_agent(pml + 2 * (sp * G + g)), l = lc_load_agent(pml + 2 * (sp * G + g) + 1);
        ph.merge.scale[half][sp] = m;
        ph.merge.sum[half][sp] = l;
        m_all = fmaxf(m_all, m);
    }
    m_all = fmaxf(m_all, lc_dpp<0xB1>(m_all));
    m_all = fmaxf(m_all, lc_dpp<0x4E>(m_all));
    m_all = fmaxf(m_all, lc_dpp<0x141>(m_all));
    m_all = fmaxf(m_all, lc_dpp<0x140>(m_all));
    {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(m_all), __float_as_uint(m_all), false, false);
        m_all = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    const float ref = m_all == LC_NEG_INF ? 0.f : m_all;
    const int n_slots = (S_eff + 8 * WAYS - 1) / (8 * WAYS) * (8 * WAYS);
    for (int sp = hl; sp < n_slots; sp += 32) {              // (this lane's own entries; up to the end of the last round, where sums are zero)
        const float f = sp >= S_eff ? 0.f : __builtin_amdgcn_exp2f((sp < 32 ? m0 : ph.merge.scale[half][sp]) - ref);
        if (sp < S_eff) den = fmaf(sp < 32 ? l0 : ph.merge.sum[half][sp], f, den);
        ph.merge.scale[half][sp] = f;
    }
    den = lc_sum16(den);
    den = lc_add_rows(den, den);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
    if (wy < WAYS) {
        for (int sp0 = 0; sp0 < S_eff; sp0 += MR * WAYS) {
            if (sp0 != 0) load_round(sp0);
#pragma unroll
            for (int k0 = 0; k0 < MR; k0 += 8)
                if (sp0 + k0 * WAYS < S_eff) {
#pragma unroll
                    for (int k = k0; k < k0 + 8; ++k) {
                        const float f = ph.merge.scale[half][sp0 + wy + k * WAYS];
                        num.x = fmaf(x[k].x, f, num.x); num.y = fmaf(x[k].y, f, num.y);
                        num.z = fmaf(x[k].z, f, num.z); num.w = fmaf(x[k].w, f, num.w);
                    }
                }
        }
    }
    if (WAYS > 1) {
        if (wy > 0 && wy < WAYS) ph.merge.red[(wy - 1) * NV + v] = num;
        __syncthreads();
    }
    if (wy == 0) {
#pragma unroll
        for (int k = 1; k < WAYS; ++k) {
            const float4 o = ph.merge.red[(k - 1) * NV + v];
            num.x += o.x; num.y += o.y; num.z += o.z; num.w += o.w;
        }
        finish(g, c4, num, ref, den);
    }
    if (tid == 0) ix.sync[bh * 4 + 1] = 0;
}

template <int G>
int launch_decode4(const LcDecode4Args& a, int splits, hipStream_t stream) {
    hipLaunchKernelGGL((lc_decode4_kernel<G>), dim3(a.ix.H, a.ix.B, splits), dim3(LC_D4_THREADS), 0, stream, a);
    LC_HIP_CHECK(hipGetLastError());
    return LC_OK;
}

// ---------------------------------------------------------------- arguments
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int check_strides16(const int64_t s[3]) {
    if (!s) return LC_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || s[i] % 8 != 0) return LC_ERR_BAD_SHAPE;
    return s[2] < LC_HEAD_DIM ? LC_ERR_BAD_SHAPE : LC_OK;
}

// Rows of all sequences of a store or load, LC_C4_BATCH sequences to a launch.
int move_rows(bool store, const void* K, const void* V, const int64_t s[3], const int32_t* first, const int32_t* counts, int B, int H_kv, int d,
              const void* K4, const void* V4, const int64_t s4[3], int max_tokens, hipStream_t stream) {
    if (!counts || !K4 || !V4 || B < 1 || H_kv < 1 || max_tokens < 1) return LC_ERR_INVALID_ARG;
    int longest = 0;
    for (int b = 0; b < B; ++b) longest = counts[b] > longest ? counts[b] : longest;
    if (longest > 0 && (!K || !V)) return LC_ERR_INVALID_ARG;               // (a tensor without rows has no address)
    if (d != LC_HEAD_DIM || H_kv > 65535) return LC_ERR_BAD_SHAPE;
    int rc = check_strides16(s);
    if (rc == LC_OK) rc = lc_check_strides4(s4);
    if (rc) return rc;
    if (!aligned(K, 16) || !aligned(V, 16) || !aligned(K4, 4) || !aligned(V4, 4)) return LC_ERR_INVALID_ARG;
    for (int b = 0; b < B; ++b) {
        if (counts[b] < 0 || (first && first[b] < 0)) return LC_ERR_INVALID_ARG;
        if ((long long)counts[b] + (first ? first[b] : 0) > max_tokens) return LC_ERR_CAPACITY;
    }
    for (int b0 = 0; b0 < B; b0 += LC_C4_BATCH) {
        LcMove4Args a;
        const int nb = B - b0 < LC_C4_BATCH ? B - b0 : LC_C4_BATCH;
        a.K = static_cast<uint16_t*>(const_cast<void*>(K)) + b0 * s[0];
        a.V = static_cast<uint16_t*>(const_cast<void*>(V)) + b0 * s[0];
        a.K4 = static_cast<uint8_t*>(const_cast<void*>(K4)) + b0 * s4[0];
        a.V4 = static_cast<uint8_t*>(const_cast<void*>(V4)) + b0 * s4[0];
        a.seq = s[0]; a.head = s[1]; a.tok = s[2];
        a.seq4 = s4[0]; a.head4 = s4[1]; a.tok4 = s4[2];
        int most = 0;
        for (int i = 0; i < LC_C4_BATCH; ++i) {
            a.r.first[i] = i < nb && first ? first[b0 + i] : 0;
            a.r.count[i] = i < nb ? counts[b0 + i] : 0;
            if (a.r.count[i] > most) most = a.r.count[i];
        }
        if (most == 0) continue;
        const dim3 grid((most + LC_C4_ROWS - 1) / LC_C4_ROWS, H_kv, 2 * nb);
        if (store) hipLaunchKernelGGL(lc_store4_kernel, grid, dim3(LC_C4_THREADS), 0, stream, a);
        else hipLaunchKernelGGL(lc_load4_kernel, grid, dim3(LC_C4_THREADS), 0, stream, a);
        LC_HIP_CHECK(hipGetLastError());
    }
    return LC_OK;
}

}  // namespace

int lc_check_strides4(const int64_t s[3]) {
    if (!s) return LC_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || s[i] % 4 != 0) return LC_ERR_BAD_SHAPE;
    return s[2] < LC_ROW4 ? LC_ERR_BAD_SHAPE : LC_OK;
}

extern "C" {

int lc_cache4_store(const void* K, const void* V, const int64_t kv_strides[3], const int32_t* first, const int32_t* counts, int B, int H_kv, int d,
                    void* K4, void* V4, const int64_t strides4[3], int max_tokens, void* stream) {
    return move_rows(true, K, V, kv_strides, first, counts, B, H_kv, d, K4, V4, strides4, max_tokens, static_cast<hipStream_t>(stream));
}

int lc_cache4_load(const void* K4, const void* V4, const int64_t strides4[3], const int32_t* first, const int32_t* counts, int B, int H_kv, int d,
                   void* K, void* V, const int64_t kv_strides[3], int max_tokens, void* stream) {
    return move_rows(false, K, V, kv_strides, first, counts, B, H_kv, d, K4, V4, strides4, max_tokens, static_cast<hipStream_t>(stream));
}

int lc_sparse_decode4(const lc_index* idx, const void* q, const void* K4, const void* V4, const int64_t strides4[3],
                      const int32_t* chunk_ids, const int32_t* counts, int cap, int H_q, float* out, float* lse,
                      void* ws, size_t ws_bytes, void* stream) {
    if (!idx || !q) return LC_ERR_INVALID_ARG;
    if (H_q < idx->H_kv || H_q % idx->H_kv != 0 || H_q / idx->H_kv > LC_MAX_GROUP) return LC_ERR_BAD_SHAPE;
    if (cap < 1 || !K4 || !V4 || !chunk_ids || !counts || !out || !ws) return LC_ERR_INVALID_ARG;
    const int rc = lc_check_strides4(strides4);
    if (rc) return rc;
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(K4, 4) || !aligned(V4, 4) || !aligned(ws, 256)) return LC_ERR_INVALID_ARG;
    const int G = H_q / idx->H_kv;
    int splits = lc_auto_splits(&idx->cfg, idx->B, idx->H_kv);
    if (ws_bytes < lc_layout_ws(&idx->cfg, idx->B, H_q, idx->H_kv, idx->d, splits, nullptr, nullptr, false)) return LC_ERR_WORKSPACE_TOO_SMALL;
    // the kernel addresses the rows of one (sequence, head) with 32-bit byte offsets
    if ((long long)idx->cfg.max_tokens * strides4[2] >= (1LL << 31) - 128) return LC_ERR_BAD_SHAPE;
    LcWs w;
    lc_layout_ws(&idx->cfg, idx->B, H_q, idx->H_kv, idx->d, splits, ws, &w, false);
    LcDecode4Args a;
    a.ix = idx->dev;
    a.q = static_cast<const uint16_t*>(q);
    a.K = static_cast<const uint8_t*>(K4);
    a.V = static_cast<const uint8_t*>(V4);
    a.seq = strides4[0]; a.head = strides4[1]; a.tok = (int)strides4[2];
    a.max_tokens = idx->cfg.max_tokens;
    a.ids = chunk_ids;
    a.counts = counts;
    a.cap = cap;
    a.part_acc = w.part_acc;
    a.part_ml = w.part_ml;
    a.out = out;
    a.lse = lse;
    // splits that can find work at the index's length (the others would only read the list)
    int most = 1;
    for (int b = 0; b < idx->B; ++b) most = idx->T[b] > most ? idx->T[b] : most;
    const int useful = (most + LC_D4_MIN_TOKENS - 1) / LC_D4_MIN_TOKENS;
    if (useful < splits) splits = useful;
    hipStream_t st = static_cast<hipStream_t>(stream);
    switch (G) {
        case 1: return launch_decode4<1>(a, splits, st);
        case 2: return launch_decode4<2>(a, splits, st);
        case 3: return launch_decode4<3>(a, splits, st);
        case 4: return launch_decode4<4>(a, splits, st);
        case 5: return launch_decode4<5>(a, splits, st);
        case 6: return launch_decode4<6>(a, splits, st);
        case 7: return launch_decode4<7>(a, splits, st);
        default: return launch_decode4<8>(a, splits, st);
    }
}

int lc_append4(lc_index* idx, void* K4, void* V4, const int64_t strides4[3], const void* k_new, const void* v_new,
               const uint8_t* close_chunk, void* stream) {
    if (!idx || !K4 || !V4 || !k_new || !v_new) return LC_ERR_INVALID_ARG;
    int rc = lc_check_strides4(strides4);
    if (rc) return rc;
    if (!aligned(K4, 4) || !aligned(V4, 4) || !aligned(k_new, 16) || !aligned(v_new, 16)) return LC_ERR_INVALID_ARG;
    if (idx->B > 1024) return LC_ERR_CAPACITY;
    for (int b = 0; b < idx->B; ++b) {
        if (idx->T[b] + 1 > idx->cfg.max_tokens) return LC_ERR_CAPACITY;
        if (close_chunk && close_chunk[b] && idx->M[b] + 1 > idx->cfg.max_chunks) return LC_ERR_CAPACITY;
    }
    rc = lc_launch_append4(idx, K4, V4, strides4, k_new, v_new, close_chunk, static_cast<hipStream_t>(stream));
    if (rc != LC_OK) return rc;
    for (int b = 0; b < idx->B; ++b) {
        idx->T[b] += 1;
        idx->tail[b] += 1;
        if (close_chunk && close_chunk[b]) {
            idx->tail[b] = 0;
            idx->M[b] += 1;
            idx->N[(size_t)b * LC_MAX_LEVELS + 0] = idx->M[b];
        }
    }
    return LC_OK;
}

}  // extern "C"
