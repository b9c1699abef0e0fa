// Attention over the key blocks that a bit mask gives each block of queries.
//
// bf16: one pass over the keys, exponentials against a reference score.  A wave takes 64 (or 32) queries of one query block and walks its list of
// key blocks in steps of 32 keys.  Scores are computed transposed (S^T = K Q^T), so that a lane owns one query column: a reference needs one
// exchange between the halves of a wave, and the probabilities are where the second product (O^T = V^T P^T) wants them.  A block that is not
// chosen is never read.
// fp32: a workgroup takes 16 queries, its four waves the steps in turn, each with a softmax of its own; joined through LDS.
#include <type_traits>
#include <utility>

#include "common.h"

namespace drf {

namespace {

typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
#define DRF_LDS_PTR __attribute__((address_space(3)))

constexpr int kMaxD = 128, kStep = 32;

struct Rows { const void* p; int64_t slot, token, head; };

struct BlockArgs {
    Rows q, k, v;
    void* out; int64_t out_slot, out_token, out_head;
    const uint32_t* blocks;
    const int32_t *q_lens, *kv_lens;
    int slots, nq, nk, q_heads, group, d;       // group: query heads a kv head
    int q_shift, kv_shift, q_blocks, words;     // log2 of the block sizes
    float scale_log2;                           // log2(e) * scale
    int split;                                  // workgroups to a tile, where four waves share it; more than one: they leave their part in `parts`
    float* parts;                               // [tile][split][32][d + 4]: O, and m and l behind it
};

// The steps of 32 keys of a query block's list, W of them passed over after each.  All of it is scalar arithmetic.
template <int W> struct Walk {
    typedef const __attribute__((address_space(4))) uint32_t* scalar_ptr;
    scalar_ptr row; uint32_t last_mask; int words, len, shift, w = -1, base = 0, sub, skip; uint32_t bits = 0;
    __device__ Walk(const BlockArgs& a, int slot, int h, int q0, int len_, int first)
        : row((scalar_ptr)(uintptr_t)(a.blocks + (((size_t)slot * a.q_heads + h) * a.q_blocks + (q0 >> a.q_shift)) * a.words)), len(len_), shift(a.kv_shift), skip(first)
    {
        const int valid = (len + (1 << shift) - 1) >> shift;    // key blocks that hold a key; bits behind them do not count
        words = (valid + 31) >> 5;
        last_mask = valid & 31 ? (1u << (valid & 31)) - 1 : ~0u;
        sub = 1 << (shift - 5);
    }
    // first key of the next step; -1: none
    __device__ int next()
    {
        for (;;) {
            if (sub == 1 << (shift - 5)) {
                while (bits == 0) {
                    if (w + 1 >= words) return -1;
                    ++w;
                    bits = row[w] & (w + 1 == words ? last_mask : ~0u);
                }
                base = (32 * w + __builtin_ctz(bits)) << shift;
                bits &= bits - 1;
                sub = 0;
            }
            const int kv0 = base + kStep * sub;
            if (kv0 >= len) { sub = 1 << (shift - 5); continue; }           // the last block ends before its last step
            ++sub;
            if (W == 1 || skip-- == 0) { skip = W - 1; return kv0; }
        }
    }
};

// The same of one in `every`, past whole words and blocks of them at once.  (Apart, since its few instructions more cost the other 5 to 10 %.)
struct WalkOfParts {
    Walk<1>::scalar_ptr row; uint32_t last_mask; int words, len, shift, w = -1, base = 0, sub, skip, every; uint32_t bits = 0;
    __device__ WalkOfParts(const BlockArgs& a, int slot, int h, int q0, int len_, int first, int every_) : skip(first), every(every_)
    {
        const Walk<1> all(a, slot, h, q0, len_, 0);
        row = all.row; last_mask = all.last_mask; words = all.words; len = all.len; shift = all.shift; sub = all.sub;
    }
    __device__ int next()
    {
        const int n = 1 << (shift - 5);                         // steps of a block; those that the last block has not count too (none follows)
        for (;;) {
            if (sub == n) {
                while (bits == 0) {
                    if (w + 1 >= words) return -1;
                    ++w;
                    bits = row[w] & (w + 1 == words ? last_mask : ~0u);
                }
                const int all = __builtin_popcount(bits) * n;
                if (skip >= all) { skip -= all; bits = 0; continue; }
                for (; skip >= n; skip -= n) bits &= bits - 1;
                base = (32 * w + __builtin_ctz(bits)) << shift;
                bits &= bits - 1;
                sub = 0;
            }
            const int kv0 = base + kStep * sub;
            if (kv0 >= len) { sub = n; continue; }
            ++sub;
            if (skip-- == 0) { skip = every - 1; return kv0; }
        }
    }
};

// Shapes that follow from the head width d = 8 P8.
template <int P8> struct Cfg {
    static constexpr int d = P8 * 8, KS = (P8 + 1) / 2;
    static constexpr bool TAIL = d % 32 == 8;                   // the last 8 rows of O^T and the denominator: one 16-row tile
    static constexpr int DT = TAIL ? d / 32 : (d + 31) / 32, DT1 = DT > 0 ? DT : 1;     // 32-row tiles of O^T
    static constexpr bool ONES = d % 32 != 0;                   // O^T has a padding row: it accumulates the denominator
    static constexpr int KP = P8 | 1;                           // 16-byte pieces per K row in LDS: odd, rows on different banks
    // and per V row: two modulo four, which keeps the four rows of a transposing read half apart (34 to 38 % of the LDS cycles are still conflicts, widths 72
    // and 128; 20 pieces a row of 128 have none and are 1 - 2 % slower, for what they add to the copies)
    static constexpr int VP = P8 + (P8 % 4 == 2 ? 0 : P8 % 4 == 3 ? 3 : 2 - P8 % 4);
    static constexpr int KI = (kStep * KP + 63) / 64, VI = (kStep * VP + 63) / 64;      // copy instructions a step
    static constexpr int KBYTES = kStep * KP * 16, BUF = KBYTES + kStep * VP * 16;
    // 16 bytes of zeros: K in the spare columns of the last k-step, V in those behind the head width but for the first, which is one: 1, 0, 0, 0
    static constexpr int ZERO = 2 * BUF, ONE = ZERO + 16;
    static constexpr int LDO = DT * 32 + (TAIL ? 16 : 0) + 8;   // row stride of an output tile
    static constexpr int WAVE = ONE + 16;                       // LDS of a wave
    static_assert(32 * LDO * 2 <= WAVE, "LDS layout");
    static constexpr int JOIN = 32 * (d + 4) * 4;               // a wave's share of O and its m and l, where waves share a tile
};

// 64 pieces of 16 bytes, lane i's from src + off to byte 16 i behind dst (LOW: only those of lanes 0 .. 31).  Every lane of the wave is active here.
template <bool LOW> __device__ inline void copy_pieces(uint32_t dst, uint32_t off, const bf16_t* src)
{
    if constexpr (LOW) asm volatile("s_mov_b32 m0, %0\n\ts_mov_b32 exec_hi, 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 exec_hi, -1" :: "s"(dst), "v"(off), "s"(src) : "memory");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(dst), "v"(off), "s"(src) : "memory");
}

// The same for the lanes of two scalar masks.
__device__ inline void copy_pieces_of(uint32_t low, uint32_t high, uint32_t dst, uint32_t off, const bf16_t* src)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %4\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b64 exec, -1"
                 :: "s"(dst), "v"(off), "s"(src), "s"(low), "s"(high) : "memory");
}

constexpr float kTau = 8.f;                                     // lazy-rescale headroom of the online softmax, in log2 units
constexpr float kNone = -3.4028235e38f;                         // no reference score yet
constexpr float kFar = 1.8446744e19f;                           // 2^64: sums up to here (of a reference of weight 1) have lost nothing
constexpr float kLargeReference = 1048576.f;                    // 2^20: a reference below is an exponent of two within 2^-4

__device__ inline float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }

// A wave owns 32 QB queries, walks its own list and stages K and V for itself alone: nothing is shared, so no wave waits for another's list, and
// the only waits are for the copies of a step that were asked for a whole step before.  Two buffers of 32 keys: while a step is computed the
// fragments of the next are read out of one and the step after it lands in the other.  With QB = 2 every fragment is used twice and one
// block's scores are formed beside the other's exponentials.  W waves share a tile of queries where there are few (each takes every W-th
// step; joined through LDS).  SH = 2 waves, of 64 queries of one block each, share its list and the buffers (one copies K, the other V), with a
// barrier where a buffer has landed and one where it is free.
// Bound by the matrix instructions and, beside them, the exponentials and the way of K and V into LDS: 4 slots x 16384 queries x 12 heads of 128
// over 16 of 128 blocks of 128, 825 GFLOP, 0.89 ms, 0.93 PFLOP/s (a large library product reaches 1.23 here, the instruction by itself 1.94; by
// waves of their own 0.94 ms, of which the copies were 0.2 and their waits nothing).  6 x 4096 x 16 of 72 over 8 of 64 blocks of 64, 58 GFLOP over
// 226 MB of q, k, v and result, 83 us, 97 with nothing of them in the caches: 24 us and 7.4 a block (1 block 34, 2 43, 4 54, 16 143, 32 263).
template <int P8, int QB, int W, int SH, bool SPLIT>
__global__ void __launch_bounds__(64 * W * SH, P8 > 11 && QB == 2 ? 1 : 2) block_attn_kernel(const BlockArgs a, int q_tiles, int n_items)
{
    using C = Cfg<P8>;
    constexpr int d = C::d, KS = C::KS, DT = C::DT, DT1 = C::DT1, KP = C::KP, VP = C::VP, LDO = C::LDO;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    static_assert(SH == 1 || (W == 1 && QB == 2), "two waves of 64 queries share their keys");
    const int wave = W * SH > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    unsigned char* mem = smem + (SH > 1 ? 0 : wave * C::WAVE);
    int item = item_by_xcd(blockIdx.x, n_items);                // query tiles of one head on one XCD
    const int part = SPLIT ? item % a.split : 0;
    if (SPLIT) item /= a.split;
    const int tile = item % q_tiles, sh = item / q_tiles, slot = sh / a.q_heads, h = sh - slot * a.q_heads;
    const int tile_q0 = tile * 32 * QB * SH, q_len = slot_len(a.q_lens, slot, a.nq), kv_len = slot_len(a.kv_lens, slot, a.nk);
    if (tile_q0 >= q_len) return;
    const int q0 = tile_q0 + (SH > 1 ? wave * 32 * QB : 0);     // (of two waves the second's queries may all lie behind the last: it works for the first)
    const bf16x8 zero8 = { 0, 0, 0, 0, 0, 0, 0, 0 };
    const bf16_t* Q = (const bf16_t*)a.q.p + slot * a.q.slot + h * a.q.head;
    const bf16_t* K = (const bf16_t*)a.k.p + slot * a.k.slot + h / a.group * a.k.head;
    const bf16_t* V = (const bf16_t*)a.v.p + slot * a.v.slot + h / a.group * a.v.head;
    const int ldk = (int)a.k.token, ldv = (int)a.v.token;

    auto walk = [&] {
        if constexpr (SPLIT) return WalkOfParts(a, slot, h, tile_q0, kv_len, part * W + wave, a.split * W);
        else return Walk<W>(a, slot, h, tile_q0, kv_len, W > 1 ? wave : 0);
    }();
    const uint32_t lds = (uint32_t)(uintptr_t)(DRF_LDS_PTR unsigned char*)mem;
    // of a lane's pieces from the step's first row (pieces of row padding take any); of two waves the first copies K, the second V
    constexpr int MOST = C::KI > C::VI ? C::KI : C::VI, COPIES = SH > 1 ? MOST : C::KI + C::VI;
    uint32_t ko[SH > 1 ? 1 : C::KI], vo[SH > 1 ? MOST : C::VI];
    const bool copies_k = SH > 1 && wave == 0;
    auto offsets = [&](int left) {
        int l = lane;
        asm volatile("" : "+v"(l));                             // formed anew each time: the lane's parts of it need no registers in between
        if constexpr (SH > 1) {
            if (copies_k) {
#pragma unroll
                for (int i = 0; i < MOST; ++i) {
                    const int id = i * 64 + l, r = id / KP, c = id % KP;
                    vo[i] = (uint32_t)((r < left ? r : left - 1) * ldk + (c < P8 ? c : 0) * 8) * 2u;
                }
            } else {
#pragma unroll
                for (int i = 0; i < MOST; ++i) {
                    const int id = i * 64 + l, r = id / VP, c = id % VP;
                    vo[i] = (uint32_t)((r < left ? r : left - 1) * ldv + (c < P8 ? c : 0) * 8) * 2u;
                }
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < (SH > 1 ? 0 : C::KI); ++i) {
            const int id = i * 64 + l, r = id / KP, c = id % KP;
            ko[i] = (uint32_t)((r < left ? r : left - 1) * ldk + (c < P8 ? c : 0) * 8) * 2u;
        }
#pragma unroll
        for (int i = 0; i < C::VI; ++i) {
            const int id = i * 64 + l, r = id / VP, c = id % VP;
            vo[i] = (uint32_t)((r < left ? r : left - 1) * ldv + (c < P8 ? c : 0) * 8) * 2u;
        }
    };
    offsets(kStep);
    // keys behind the last repeat it (see tail): the last step of the list only
    auto next_step = [&]() {
        const int kv0 = walk.next();
        if (kv0 >= 0 && kv_len - kv0 < kStep) offsets(kv_len - kv0);
        return kv0;
    };
    // copy j of the step at kv0
    const int ldc = copies_k ? ldk : ldv;
    const bf16_t* const from = copies_k ? K : V;
    auto copy = [&](int kv0, int buf, int j) {
        const uint32_t b = lds + (uint32_t)buf * C::BUF;
        if constexpr (SH > 1) {
            const bf16_t* src = from + (int64_t)kv0 * ldc;
            const uint32_t dst = b + (copies_k ? 0u : (uint32_t)C::KBYTES) + j * 1024u;
            // (rows come in 32s: a last copy is of half a wave or a whole one)
            const int left_k = kStep * KP - 64 * j, left_v = kStep * VP - 64 * j;
            if (left_k >= 64 && left_v >= 64) {
                copy_pieces<false>(dst, vo[j], src);
            } else {
                const int left = copies_k ? left_k : left_v;
                copy_pieces_of(__builtin_amdgcn_readfirstlane(left > 0 ? -1 : 0), __builtin_amdgcn_readfirstlane(left >= 64 ? -1 : 0), dst, vo[j], src);
            }
        } else if (j < C::KI) {
            const bf16_t* src = K + (int64_t)kv0 * ldk;
            if (j == C::KI - 1 && kStep * KP % 64) copy_pieces<true>(b + j * 1024u, ko[j], src);
            else copy_pieces<false>(b + j * 1024u, ko[j], src);
        } else {
            const bf16_t* src = V + (int64_t)kv0 * ldv;
            const int i = j - C::KI;
            if (i == C::VI - 1 && kStep * VP % 64) copy_pieces<true>(b + C::KBYTES + i * 1024u, vo[i], src);
            else copy_pieces<false>(b + C::KBYTES + i * 1024u, vo[i], src);
        }
    };
    auto issue = [&](int kv0, int buf) {
#pragma unroll
        for (int j = 0; j < COPIES; ++j) copy(kv0, buf, j);
    };
    // every copy has landed, every LDS read is done
    auto settle_memory = [&]() {
        if constexpr (SH > 1) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    };
    // values behind the last key of a landed step that the keys end inside of are zero, not repeated (a weight of zero takes no NaN with it)
    auto tail = [&](int kv0, int buf) {
        const int left = kv_len - kv0;
        if (left < kStep)
            for (int i = left * VP + lane; i < kStep * VP; i += 64) *reinterpret_cast<bf16x8*>(mem + buf * C::BUF + C::KBYTES + i * 16) = zero8;
    };

    int n0 = next_step(), n1 = -1;
    if (n0 >= 0) {
        issue(n0, 0);
        n1 = next_step();
        if (n1 >= 0) issue(n1, 1);
    }
    if (lane < 2) {
        bf16x8 v = zero8;
        if (lane == 1) v[0] = (bf16_t)1.f;
        *reinterpret_cast<bf16x8*>(mem + C::ZERO + lane * 16) = v;
    }
    bf16x8 qf[QB][KS];
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int q = q0 + b * 32 + l32 < q_len ? q0 + b * 32 + l32 : q_len - 1;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int c = ks * 16 + half * 8;
            qf[b][ks] = c < d ? *reinterpret_cast<const bf16x8*>(Q + (int64_t)q * a.q.token + c) : zero8;
        }
    }
#pragma unroll
    for (int b = 0; b < QB; ++b)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[b][ks]));

    f32x16 o[QB][DT1];
    f32x4 ot[QB][2];                                            // TAIL: rows 32 DT .. 32 DT + 15, queries 0-15 and 16-31 of block b
    // Exponents are taken against a reference score m_run; ms: it, in exponents of two where it stays (0 while there is none: then every score so far is
    // -infinity).
    const float sl2 = a.scale_log2, tau = kTau / sl2;
    float m_run[QB], ms[QB], l_run[QB];

    bf16x8 kf[KS], vf[2][DT1], vt, pf[QB][2];
    f32x16 s[QB];
    const f32x16 zero16 = { 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f };
    const int koff = l32 * KP * 8 + half * 8;
    const int voff = C::KBYTES / 2 + (4 * half + ((lane & 15) >> 2)) * VP * 8 + (l32 & 16) + 4 * (lane & 3);
    // tail tile: k-slices of the 16 x 16 x 32 product are (rows 0-15, half 0), (16-31, 0), (0-15, 1), (16-31, 1), see pv
    const int voff_t = C::KBYTES / 2 + (16 * ((lane >> 4) & 1) + 4 * half + ((lane & 15) >> 2)) * VP * 8 + DT * 32 + 4 * (lane & 3);
    // where this lane's four columns of the last tile lie behind the head width: one, then zeros
    const int last_col = C::TAIL ? DT * 32 + 4 * (lane & 3) : (DT - 1) * 32 + (l32 & 16) + 4 * (lane & 3);
    const bf16_t* spare = reinterpret_cast<const bf16_t*>(mem + (last_col == d ? C::ONE : C::ZERO));
    auto load_k = [&](int buf) {
        const bf16_t* p = reinterpret_cast<const bf16_t*>(mem + buf * C::BUF) + koff;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const bf16_t* pk = p + ks * 16;
            if (P8 % 2 == 1 && ks == KS - 1) pk = half ? reinterpret_cast<const bf16_t*>(mem + C::ZERO) : pk;
            kf[ks] = *reinterpret_cast<const bf16x8*>(pk);
        }
    };
    // lane i of 16 receives column i of 4 rows, and of the 4 rows 8 further on; in the last tile that has columns behind the head width, those from `spare`
    auto transposed = [&](const bf16_t* p, bool last) {
        const bf16_t* p8 = p + 8 * VP * 8;
        if (C::ONES && last) {
            p = last_col >= d ? spare : p;
            p8 = last_col >= d ? spare : p8;
        }
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((DRF_LDS_PTR s16x4*)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((DRF_LDS_PTR s16x4*)p8);
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto load_v = [&](int buf) {
        const bf16_t* p = reinterpret_cast<const bf16_t*>(mem + buf * C::BUF);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int t = 0; t < DT; ++t) vf[c][t] = transposed(p + voff + 16 * c * VP * 8 + t * 32, !C::TAIL && t == DT - 1);
        if constexpr (C::TAIL) vt = transposed(p + voff_t, true);
    };
    // `after`: called behind each matrix instruction with its number
    auto nothing = [](int) {};
    auto qk = [&](int b, auto after) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[b][ks], ks == 0 ? zero16 : s[b], 0, 0, 0);
            after(ks);
        }
    };
    // register r of s[b] holds key 8 (r / 4) + 4 half + r % 4 of a step: keys behind the last score -infinity
    auto mask = [&](int b, int kv0) {
        if (kv_len - kv0 < kStep) {
            const int left = kv_len - kv0 - 4 * half;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r >> 2) + (r & 3) >= left) s[b][r] = -INFINITY;
        }
    };
    auto largest = [&](int b) {                                 // of this lane's scores
        float mx = max3(s[b][0], s[b][1], s[b][2]);
#pragma unroll
        for (int r = 3; r < 15; r += 2) mx = max3(mx, s[b][r], s[b][r + 1]);
        return __builtin_elementwise_maximum(mx, s[b][15]);
    };
    auto refer = [&](auto lazy_c, int b, float mx) {            // to the largest of both halves' scores if that is more
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        m_run[b] = max3(__uint_as_float(sw[0]), __uint_as_float(sw[1]), m_run[b]);
        ms[b] = m_run[b] == kNone ? 0.f : decltype(lazy_c)::value ? m_run[b] : m_run[b] * sl2;
    };
    // The reference moves only when some query of the block would otherwise exceed 2^kTau, or has none yet and a score to refer to (which may be the
    // lowest number, and tau as large as the largest).
    auto settle = [&](int b) {
        const float mx = largest(b);
        if (__any(mx - m_run[b] >= tau || (m_run[b] == kNone && mx > kNone))) {
            const float old = m_run[b];
            refer(std::true_type{}, b, mx);
            const float alpha = __builtin_amdgcn_exp2f((old - m_run[b]) * sl2);
            l_run[b] *= alpha;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[b][t][r] *= alpha;
            if constexpr (C::TAIL) {                            // here a lane's query is lane % 16 (+ 16)
                const auto al = __builtin_amdgcn_permlane16_swap(__float_as_uint(alpha), __float_as_uint(alpha), false, false);
#pragma unroll
                for (int r = 0; r < 4; ++r) { ot[b][0][r] *= __uint_as_float(al[0]); ot[b][1][r] *= __uint_as_float(al[1]); }
            }
        }
    };
    // P of block b, rounded to bf16 for the matrix instruction (its fp32 form has a sixteenth of the rate): half a step of a weight at most, which takes
    // the error of a result from 0.0017 of its size, what its own rounding leaves, to 0.0018.  The denominator sums the weights before that rounding
    // where the head width is a multiple of 32, and in the matrix instruction, after it, where O^T has a row to spare.
    // LAZY takes the difference first, which is exact where it matters, whatever the scores' size (0.2 us of a query's 10.3 over 1024 keys; by a
    // branch for large references alone 0.3); otherwise one instruction does, and what the reference's rounding to an exponent of two leaves (2^-24 of it) is
    // common to a query's weights.
    auto soft = [&](auto lazy_c, int b) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = s[b][8 * c + e];
                s[b][8 * c + e] = __builtin_amdgcn_exp2f(decltype(lazy_c)::value ? (x - ms[b]) * sl2 : fmaf(x, sl2, -ms[b]));
            }
            if constexpr (!C::ONES) {
#pragma unroll
                for (int e = 0; e < 8; ++e) l_run[b] += s[b][8 * c + e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) pf[b][c][e] = (bf16_t)s[b][8 * c + e];
        }
    };
    // O^T[d][q] += sum over keys V^T[d][key] P^T[key][q], 16 keys (8 of a lane's scores) at a time
    auto pv = [&](int b, auto after) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                o[b][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[c][t], pf[b][c], o[b][t], 0, 0, 0);
                after(c * DT + t);
            }
        if constexpr (C::TAIL) {
            // 16 x 16 x 32 operands of queries 0-15 and 16-31: rows of 16 lanes 1, 3 of the first chunk against 0, 2 of the second
            u32x4 p0 = __builtin_bit_cast(u32x4, pf[b][0]), p1 = __builtin_bit_cast(u32x4, pf[b][1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const auto sw = __builtin_amdgcn_permlane16_swap(p0[i], p1[i], false, false);
                p0[i] = sw[0]; p1[i] = sw[1];
            }
            ot[b][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8, p0), ot[b][0], 0, 0, 0);
            ot[b][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, __builtin_bit_cast(bf16x8, p1), ot[b][1], 0, 0, 0);
        }
    };
    auto pin = []() { __builtin_amdgcn_sched_barrier(0x40f); };             // LDS accesses stay on their side, the rest may cross

    // The whole list, whose first two steps are on their way.  LAZY: the reference follows the scores; otherwise it is the largest of the first
    // step's, and the straight line of a step has neither maxima nor a branch in it.
    auto run = [&](auto lazy_c, int n0, int n1) {
        constexpr bool LAZY = decltype(lazy_c)::value;
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            m_run[b] = kNone; ms[b] = 0.f; l_run[b] = 0.f;
#pragma unroll
            for (int t = 0; t < DT; ++t) o[b][t] = zero16;
            ot[b][0] = ot[b][1] = (f32x4){ 0.f, 0.f, 0.f, 0.f };
        }
        if (n0 < 0) return;
        settle_memory();
        tail(n0, 0);
        if (n1 >= 0) tail(n1, 1);
        load_k(0);
        if constexpr (!LAZY && QB == 2) {
            qk(1, nothing);
            mask(1, n0);
            refer(lazy_c, 1, largest(1));
        }
        qk(0, nothing);
        mask(0, n0);
        if constexpr (LAZY) settle(0);
        else refer(lazy_c, 0, largest(0));
        if constexpr (QB == 2) {                                // the first step finds nothing pending
            pf[1][0] = pf[1][1] = zero8;
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int t = 0; t < DT1; ++t) vf[c][t] = zero8;
            vt = zero8;
        }
        int buf = 0, n2 = n1 >= 0 ? next_step() : -1;
        // Step n0: its keys' fragments and block 0's scores are in registers, with the next step in the other buffer (MORE: there is one) and step n2 on
        // its way into this one once its values' fragments have left it (ISSUE: there is one; then n0 and n1 are not the last and so are full).
        // Two blocks take turns: beside the exponentials of one run the other's scores and the product of its probabilities of half a step before.
        auto step = [&](auto issue_c, auto more_c) {
            constexpr bool ISSUE = decltype(issue_c)::value, MORE = decltype(more_c)::value;
            if constexpr (MORE) {
                if constexpr (SH > 1) asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
                else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                if (!ISSUE) tail(n1, buf ^ 1);
            }
            // Matrix instruction m of the NM beside which this buffer is refilled, a copy or two behind each: all of them at once would keep the
            // wave from issuing anything else until the CU's one path to memory had taken them.
            constexpr int NM = (QB == 2 ? KS : 0) + 2 * DT, PER = NM > 0 ? NM : 1;
            auto refill = [&](int m) {
                if constexpr (ISSUE) {
                    if (m == 0) {                               // the values' fragments are out
                        if constexpr (SH > 1) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    }
#pragma unroll
                    for (int j = m * COPIES / PER; j < (m + 1) * COPIES / PER; ++j) copy(n2, buf, j);
                    __builtin_amdgcn_sched_barrier(0x406);      // vector and scalar arithmetic may cross
                }
            };
            int n3 = -1;
            if constexpr (QB == 2) {
                qk(1, nothing);
                if constexpr (MORE) load_k(buf ^ 1);
                pin();
                soft(lazy_c, 0);
                pv(1, nothing);
                load_v(buf);
                pin();
                if constexpr (!ISSUE) mask(1, n0);
                if constexpr (LAZY) settle(1);
                if constexpr (MORE) qk(0, refill);
                soft(lazy_c, 1);
                pv(0, [&](int m) { refill(KS + m); });
                if constexpr (ISSUE) n3 = next_step();
                if constexpr (MORE) {
                    if constexpr (!ISSUE) mask(0, n1);
                    if constexpr (LAZY) settle(0);
                }
            } else {
                load_v(buf);
                if constexpr (MORE) load_k(buf ^ 1);
                pin();
                soft(lazy_c, 0);
                if constexpr (NM == 0) {
                    if constexpr (ISSUE) {
                        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                        issue(n2, buf);
                    }
                }
                pv(0, refill);
                if constexpr (MORE) qk(0, nothing);
                if constexpr (ISSUE) n3 = next_step();
                if constexpr (MORE) {
                    if constexpr (!ISSUE) mask(0, n1);
                    if constexpr (LAZY) settle(0);
                }
            }
            n0 = n1; n1 = n2; n2 = n3; buf ^= 1;
        };
        while (n2 >= 0) step(std::true_type{}, std::true_type{});
        if (n1 >= 0) step(std::false_type{}, std::true_type{});
        step(std::false_type{}, std::false_type{});
        if constexpr (QB == 2) pv(1, nothing);
    };
    if constexpr (W > 1) {
        run(std::true_type{}, n0, n1);
    } else {
        run(std::false_type{}, n0, n1);
        // Scores so far above the first step's that a sum overflows (or anything that is not a number, which stays what it is), a first step
        // that was all of -infinity and so no reference, below which all others may vanish, or a reference so large that its rounding to an exponent of
        // two is no small factor: once more with a reference that follows them.
        float top = 0.f;
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            if (m_run[b] == kNone || !(fabsf(ms[b]) < kLargeReference)) top = INFINITY;
            if (!C::ONES) top = __builtin_elementwise_maximum(top, l_run[b]);
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int r = 0; r < 16; r += 2) top = max3(top, fabsf(o[b][t][r]), fabsf(o[b][t][r + 1]));
            if (C::TAIL) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; r += 2) top = max3(top, fabsf(ot[b][i][r]), fabsf(ot[b][i][r + 1]));
            }
        }
        bool again = __any(!(top < kFar));
        if constexpr (SH > 1) {                                 // for both if for one
            uint32_t* flag = reinterpret_cast<uint32_t*>(mem + C::WAVE);
            if (lane == 0) flag[wave] = again;
            settle_memory();
            again = __builtin_amdgcn_readfirstlane(flag[0] | flag[1]) != 0;
        }
        if (again) {
            walk = Walk<W>(a, slot, h, tile_q0, kv_len, 0);
            offsets(kStep);
            settle_memory();
            n0 = next_step();
            n1 = -1;
            if (n0 >= 0) {
                issue(n0, 0);
                n1 = next_step();
                if (n1 >= 0) issue(n1, 1);
            }
            run(std::true_type{}, n0, n1);
        }
    }

    auto denominator = [&](int b) {
        if constexpr (C::TAIL) {
            // row d of O^T is row 8 of the tail tile: register 0 of lanes 32-47, query lane % 16 (+ 16)
            const float l0 = __shfl(ot[b][0][0], 32 + (lane & 15), 64), l1 = __shfl(ot[b][1][0], 32 + (lane & 15), 64);
            return l32 < 16 ? l0 : l1;
        } else if constexpr (C::ONES) {
            constexpr int lr = d & 31, r = 4 * (lr >> 3) + (lr & 3), owner = (lr >> 2) & 1;
            const float mine = o[b][DT1 - 1][r], other = __shfl_xor(mine, 32, 64);
            return half == owner ? mine : other;
        } else {
            return l_run[b] + __shfl_xor(l_run[b], 32, 64);
        }
    };
    auto inverse = [](float l) { return l > 0.f ? 1.f / l : l != l ? l : 0.f; };        // no weight at all: zeros
    bf16_t* out = (bf16_t*)a.out + slot * a.out_slot + h * a.out_head;
    if constexpr (W == 1) {
        // a block's 32 x d tile is transposed through LDS, so that rows leave in 16-byte pieces (a wave's LDS operations complete in order)
        settle_memory();
        static_assert(SH * 32 * LDO * 2 <= C::WAVE, "LDS layout");
        bf16_t* so = reinterpret_cast<bf16_t*>(mem) + (SH > 1 ? wave * 32 * LDO : 0);
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            if (q0 + b * 32 >= q_len) break;
            const float inv = inverse(denominator(b));
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const bf16x4 w = { (bf16_t)(o[b][t][4 * g] * inv), (bf16_t)(o[b][t][4 * g + 1] * inv),
                                       (bf16_t)(o[b][t][4 * g + 2] * inv), (bf16_t)(o[b][t][4 * g + 3] * inv) };
                    *reinterpret_cast<bf16x4*>(so + l32 * LDO + t * 32 + 8 * g + 4 * half) = w;
                }
            if constexpr (C::TAIL) {
                if (lane < 32) {                                // rows 0-7 of the tail tile: four rows of query lane % 16 (+ 16) per lane
#pragma unroll
                    for (int qh = 0; qh < 2; ++qh) {
                        const float iv = __shfl(inv, (lane & 15) + 16 * qh, 64);
                        const bf16x4 w = { (bf16_t)(ot[b][qh][0] * iv), (bf16_t)(ot[b][qh][1] * iv),
                                           (bf16_t)(ot[b][qh][2] * iv), (bf16_t)(ot[b][qh][3] * iv) };
                        *reinterpret_cast<bf16x4*>(so + ((lane & 15) + 16 * qh) * LDO + DT * 32 + 4 * (lane >> 4)) = w;
                    }
                }
            }
            for (int id = lane; id < 32 * P8; id += 64) {
                const int r = id / P8, c = id % P8, q = q0 + b * 32 + r;
                if (q < q_len) *reinterpret_cast<bf16x8*>(out + (int64_t)q * a.out_token + c * 8) = *reinterpret_cast<const bf16x8*>(so + r * LDO + c * 8);
            }
        }
    } else {
        static_assert(W == 1 || QB == 1, "waves share tiles of 32 queries");
        // every wave leaves its O, reference and denominator; then the waves take the rows' pieces in turn
        constexpr int LDJ = d + 4;
        const float l = denominator(0);
        __syncthreads();                                        // the buffers are free
        float* mine = reinterpret_cast<float*>(smem + wave * C::JOIN);
        if (half == 0) { mine[l32 * LDJ + d] = m_run[0]; mine[l32 * LDJ + d + 1] = l; }
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (t * 32 + 8 * g + 4 * half < d)
                    *reinterpret_cast<f32x4*>(mine + l32 * LDJ + t * 32 + 8 * g + 4 * half) = (f32x4){ o[0][t][4 * g], o[0][t][4 * g + 1], o[0][t][4 * g + 2], o[0][t][4 * g + 3] };
        if constexpr (C::TAIL) {
            if (lane < 32) {
#pragma unroll
                for (int qh = 0; qh < 2; ++qh) *reinterpret_cast<f32x4*>(mine + ((lane & 15) + 16 * qh) * LDJ + DT * 32 + 4 * (lane >> 4)) = ot[0][qh];
            }
        }
        __syncthreads();
        const float* all = reinterpret_cast<const float*>(smem);
        for (int id = threadIdx.x; id < 32 * P8; id += 64 * W) {
            const int r = id / P8, c = id % P8;
            if (q0 + r >= q_len) break;
            float m = kNone, f[W], lt = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) m = __builtin_elementwise_maximum(m, all[w * (C::JOIN / 4) + r * LDJ + d]);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float mw = all[w * (C::JOIN / 4) + r * LDJ + d];
                f[w] = mw == kNone ? 0.f : __builtin_amdgcn_exp2f((mw - m) * sl2);
                lt = fmaf(all[w * (C::JOIN / 4) + r * LDJ + d + 1], f[w], lt);
            }
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = fmaf(all[w * (C::JOIN / 4) + r * LDJ + c * 8 + e], f[w], v[e]);
            if constexpr (SPLIT) {
                float* mine = a.parts + (((size_t)item * a.split + part) * 32 + r) * LDJ;
                *reinterpret_cast<f32x4*>(mine + c * 8) = (f32x4){ v[0], v[1], v[2], v[3] };
                *reinterpret_cast<f32x4*>(mine + c * 8 + 4) = (f32x4){ v[4], v[5], v[6], v[7] };
                if (c == 0) { mine[d] = m; mine[d + 1] = lt; }
            } else {
                const float inv = inverse(lt);
                bf16x8 y;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = (bf16_t)(v[e] * inv);
                *reinterpret_cast<bf16x8*>(out + (int64_t)(q0 + r) * a.out_token + c * 8) = y;
            }
        }
    }
}

// The parts of a tile's workgroups to its result: a thread 8 columns of a row.
__global__ void __launch_bounds__(256) join_parts_kernel(const BlockArgs a, int q_tiles)
{
    const int tile = blockIdx.x % q_tiles, sh = blockIdx.x / q_tiles, slot = sh / a.q_heads, h = sh - slot * a.q_heads;
    const int d = a.d, ld = d + 4, pieces = d / 8, q0 = tile * 32, q_len = slot_len(a.q_lens, slot, a.nq);
    const float* parts = a.parts + (size_t)blockIdx.x * a.split * 32 * ld;
    bf16_t* out = (bf16_t*)a.out + slot * a.out_slot + h * a.out_head;
    for (int id = threadIdx.x; id < 32 * pieces; id += 256) {
        const int r = id / pieces, c = id % pieces;
        if (q0 + r >= q_len) break;
        float m = kNone, l = 0.f, v[8] = {};
        for (int p = 0; p < a.split; ++p) m = __builtin_elementwise_maximum(m, parts[(p * 32 + r) * ld + d]);
        for (int p = 0; p < a.split; ++p) {
            const float* from = parts + (p * 32 + r) * ld;
            const float f = from[d] == kNone ? 0.f : __builtin_amdgcn_exp2f((from[d] - m) * a.scale_log2);
            const f32x4 lo = *reinterpret_cast<const f32x4*>(from + c * 8), hi = *reinterpret_cast<const f32x4*>(from + c * 8 + 4);
            l = fmaf(from[d + 1], f, l);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] = fmaf(lo[e], f, v[e]); v[4 + e] = fmaf(hi[e], f, v[4 + e]); }
        }
        const float inv = l > 0.f ? 1.f / l : l != l ? l : 0.f;
        bf16x8 y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (bf16_t)(v[e] * inv);
        *reinterpret_cast<bf16x8*>(out + (int64_t)(q0 + r) * a.out_token + c * 8) = y;
    }
}

// fp32 on the fp32 matrix instruction (16 x 16 x 4), operands straight from memory, a step's all asked for at once; DQ >= ceil(d / 16) tiles of
// columns.  Few steps: bound by the chain of a mask word, a step's rows, its products and exponentials and the join; many: by the loads' way through
// the CU's one path and the products in turn.  A lane's column of V is one of each of up to four tiles, so that they come in one load: 7 slots x
// 1000 queries x 4 heads of 32 over 5 of 32 blocks of 32 take 14.8 us (15.7 with a tile's columns side by side, 4 bytes a load), 4 x 1024 x 8 of 64
// over 4 of 16 blocks of 64 43 (50), 12 x 256 x 16 of 72 over 2 of 4 51 (64, of which 5 are columns behind the width), 2 x 4096 x 8 of 128 over 8 of
// 64 280 (312; 17.2 GFLOP).
// VEC: width, strides and addresses allow accesses of 16 bytes.
constexpr int kF32Waves = 4;
template <int DQ, bool VEC>
__global__ void __launch_bounds__(kF32Waves * 64) block_attn_f32_kernel(const BlockArgs a, int q_tiles)
{
    constexpr int E = !VEC ? 1 : DQ % 4 == 0 ? 4 : DQ % 2 == 0 ? 2 : 1;     // columns of V that a lane loads at once: one of each of E tiles
    typedef float vec __attribute__((ext_vector_type(E)));
    __shared__ float po[kF32Waves][4][DQ][64];
    __shared__ float pm[kF32Waves][16], pl[kF32Waves][16];
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = blockIdx.x % q_tiles, sh = blockIdx.x / q_tiles, slot = sh / a.q_heads, h = sh - slot * a.q_heads, d = a.d;
    const int q0 = tile * 16, q_len = slot_len(a.q_lens, slot, a.nq), kv_len = slot_len(a.kv_lens, slot, a.nk);
    if (q0 >= q_len) return;
    const int q = q0 + l16, qc = q < q_len ? q : q_len - 1;
    const float* Q = (const float*)a.q.p + slot * a.q.slot + h * a.q.head + (int64_t)qc * a.q.token;
    const float* K = (const float*)a.k.p + slot * a.k.slot + h / a.group * a.k.head;
    const float* V = (const float*)a.v.p + slot * a.v.slot + h / a.group * a.v.head;
    auto load4 = [&](const float* p, int c) -> f32x4 {          // elements c .. c + 3 of a row, zero behind its end
        f32x4 v = { 0.f, 0.f, 0.f, 0.f };
        if constexpr (VEC) {
            if (c < d) v = *reinterpret_cast<const f32x4*>(p + c);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < d) v[j] = p[c + j];
        }
        return v;
    };
    f32x4 qf[DQ], o[DQ];
#pragma unroll
    for (int c = 0; c < DQ; ++c) {
        qf[c] = load4(Q, c * 16 + 4 * quarter);
        o[c] = (f32x4){ 0.f, 0.f, 0.f, 0.f };
    }
    float m_run = -INFINITY, l_run = 0.f;                       // l_run: this quarter's share
    Walk<kF32Waves> walk(a, slot, h, q0, kv_len, wave);
    for (int kv0 = walk.next(); kv0 >= 0; kv0 = walk.next()) {
        f32x4 s[2], kf[2][DQ];
        float vf[2][4][DQ];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int row = kv0 + 16 * t + l16, rc = row < kv_len ? row : kv_len - 1;
#pragma unroll
            for (int c = 0; c < DQ; ++c) kf[t][c] = load4(K + (int64_t)rc * a.k.token, c * 16 + 4 * quarter);
        }
        // V^T operand of k-slice (t, r): key 16 t + 4 quarter + r, row l16 of tile c is column E l16 + c % E of those from 16 (c - c % E) on
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = kv0 + 16 * t + 4 * quarter + r;
#pragma unroll
                for (int c = 0; c < DQ; c += E) {
                    const int col = 16 * c + E * l16;
                    vec v = {};
                    if (row < kv_len && col < d) v = *reinterpret_cast<const vec*>(V + (int64_t)row * a.v.token + col);
#pragma unroll
                    for (int j = 0; j < E; ++j) vf[t][r][c + j] = v[j];
                }
            }
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = (f32x4){ 0.f, 0.f, 0.f, 0.f };
#pragma unroll
            for (int c = 0; c < DQ; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[t][c][j], qf[c][j], s[t], 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (kv0 + 16 * t + 4 * quarter + r >= kv_len) s[t][r] = -INFINITY;
                mx = fmaxf(mx, s[t][r]);
            }
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m_run, mx), ref = m_new == -INFINITY ? 0.f : m_new, alpha = __builtin_amdgcn_exp2f((m_run - ref) * a.scale_log2);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int c = 0; c < DQ; ++c) o[c] *= alpha;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float p = __builtin_amdgcn_exp2f((s[t][r] - ref) * a.scale_log2);
                l_run += p;
#pragma unroll
                for (int c = 0; c < DQ; ++c) o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[t][r][c], p, o[c], 0, 0, 0);
            }
    }
    l_run += __shfl_xor(l_run, 16, 64);
    l_run += __shfl_xor(l_run, 32, 64);
    if (quarter == 0) { pm[wave][l16] = m_run; pl[wave][l16] = l_run; }
#pragma unroll
    for (int c = 0; c < DQ; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) po[wave][r][c][lane] = o[c][r];
    __syncthreads();
    float m_all = pm[0][l16], l_all = 0.f, f[kF32Waves];
#pragma unroll
    for (int w = 1; w < kF32Waves; ++w) m_all = fmaxf(m_all, pm[w][l16]);
#pragma unroll
    for (int w = 0; w < kF32Waves; ++w) {                       // a wave without a score above -infinity has nothing to add
        f[w] = pm[w][l16] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((pm[w][l16] - m_all) * a.scale_log2);
        l_all += pl[w][l16] * f[w];
    }
    if (q >= q_len) return;
    const float inv = l_all > 0.f ? 1.f / l_all : l_all != l_all ? l_all : 0.f;
    float* op = (float*)a.out + slot * a.out_slot + (int64_t)q * a.out_token + h * a.out_head;
#pragma unroll
    for (int c = 0; c < DQ; c += E) {                           // wave w joins row 4 quarter + w of every tile
        const int col = 16 * c + E * (4 * quarter + wave);
        vec v;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            float x = po[0][wave][c + j][lane] * f[0];
#pragma unroll
            for (int w = 1; w < kF32Waves; ++w) x = fmaf(po[w][wave][c + j][lane], f[w], x);
            v[j] = x * inv;
        }
        if (col < d) *reinterpret_cast<vec*>(op + col) = v;
    }
}

int log2_of(int b) { return b == 32 ? 5 : b == 64 ? 6 : b == 128 ? 7 : 0; }

template <int P8, int QB, int W, int SH, bool SPLIT = false> drf_status launch_bf16_as(const BlockArgs& a, hipStream_t st)
{
    using C = Cfg<P8>;
    constexpr int smem = W * (W > 1 && C::JOIN > C::WAVE ? C::JOIN : C::WAVE) + (SH > 1 ? 16 : 0);
    static_assert(smem <= 160 * 1024, "LDS of a CU");
    auto kern = block_attn_kernel<P8, QB, W, SH, SPLIT>;
    const int q_tiles = (a.nq + 32 * QB * SH - 1) / (32 * QB * SH);
    const long long items = (long long)q_tiles * a.q_heads * a.slots * (SPLIT ? a.split : 1);
    if (items > 0x1ffffffLL / (W * SH)) DRF_FAIL(DRF_ESHAPE, "too many queries");
    static std::atomic<uint64_t> lds_allowed{ 0 };
    DRF_HIP(allow_lds(reinterpret_cast<const void*>(kern), smem, lds_allowed));
    hipLaunchKernelGGL(kern, dim3((unsigned)items), dim3(64 * W * SH), smem, st, a, q_tiles, (int)items);
    if constexpr (SPLIT) {
        DRF_HIP(hipGetLastError());
        hipLaunchKernelGGL(join_parts_kernel, dim3((unsigned)(items / a.split)), dim3(256), 0, st, a, q_tiles);
    }
    DRF_HIP(hipGetLastError());
    return DRF_OK;
}

// Workgroups to a tile of 32 queries: where the tiles leave most CUs idle and the keys are many, since one CU's way to memory (some 43 bytes a ns) then
// bounds the call.  1 query x 16 heads of 72, 8192 keys in blocks of 64, against a workgroup to a head, us: 128 blocks chosen 21.7 : 55.9, 64 15.5 : 30.0,
// 32 12.9 : 17.0, 16 11.6 : 10.5, 4 11.4 : 5.7 (the second launch and the parts).  How many are chosen only the caller knows: who gives scratch wants it.
// The rule sees the tokens alone, and below 8192 of them nothing has been measured.
int split_of(const drf_attn_shape& s)
{
    if (s.dtype != DRF_BF16) return 1;
    const long long tiles = (long long)((s.q_tokens + 31LL) / 32) * s.q_heads * s.slots;
    if (tiles == 0 || tiles > 64 || s.kv_tokens < 8192) return 1;
    const long long idle = 256 / tiles, keys = s.kv_tokens / 1024;
    return (int)(idle < keys ? idle : keys);
}

size_t parts_bytes(const drf_attn_shape& s, int split)
{
    if (split < 2) return 0;
    return (size_t)((s.q_tokens + 31LL) / 32) * s.q_heads * s.slots * split * 32 * (s.head_dim + 4) * sizeof(float);
}

// How many queries a wave takes, and whether four waves share them, by what the chip then holds at once (1024 SIMDs, 256 CUs):
//  - four waves to 32 queries while all of them fit, 8 waves to a CU or what its LDS has room for.  1 slot x 16 heads of 72, 8 blocks of 64 keys, us:
//    512 queries 7.6 against 11.3 with a wave to 32 queries and 16.1 with a wave to 64; 1024 9.3 : 11.8 : 16.3; 2048 17.3 : 13.0 : 17.5 (of 128, where four
//    waves fill a CU: 512 9.6 : 13.7 : 20.8; 1024 18.4 : 15.4 : 21.6).  Two waves are between, eight lose from 512 tiles on and gain up to 8 % before;
//  - a wave to 32 queries while that leaves no SIMD with two (2048 queries 13.0 : 17.5; of 128 18.4 : 23.9), and for query blocks of 32;
//  - a wave to 64 queries otherwise, which reads every fragment of K and V once for two blocks of queries (4096 queries 18.8 : 19.2; of 128 36.1 : 28.2;
//    6 slots x 4096 107.8 : 84.2);
//  - two such waves on one copy of the keys for query blocks of 128 and widths from 96 on, where a SIMD's registers hold one wave in any case: 4 x 16384
//    x 12 heads of 128 890 : 941, 1 x 4096 x 16 27.9 : 28.8, 2 x 8192 x 16 of 96 132 : 140.  Narrower heads have several waves to a SIMD that do better
//    without each other's waits (4 x 2048 x 8 of 64 22.9 : 18.9, of 32 39.3 : 36.6; 6 x 4096 x 16 of 72 95.7 : 99.2 the other way).
template <int P8> drf_status launch_bf16(const BlockArgs& a, hipStream_t st)
{
    constexpr int per_cu = 160 * 1024 / Cfg<P8>::WAVE < 8 ? 160 * 1024 / Cfg<P8>::WAVE : 8;
    const long long tiles = (long long)((a.nq + 31) / 32) * a.q_heads * a.slots;
    if (a.split > 1) return launch_bf16_as<P8, 1, 4, 1, true>(a, st);
    if (tiles * 4 <= 256 * per_cu) return launch_bf16_as<P8, 1, 4, 1>(a, st);
    if (tiles <= 1024 || a.q_shift == 5) return launch_bf16_as<P8, 1, 1, 1>(a, st);
    if constexpr (P8 > 11)
        if (a.q_shift == 7) return launch_bf16_as<P8, 2, 1, 2>(a, st);
    return launch_bf16_as<P8, 2, 1, 1>(a, st);
}

template <int DQ> drf_status launch_f32(const BlockArgs& a, hipStream_t st)
{
    const int q_tiles = (a.nq + 15) / 16;
    const long long items = (long long)q_tiles * a.q_heads * a.slots;
    if (items > 0x7fffffLL) DRF_FAIL(DRF_ESHAPE, "too many queries");
    auto aligned = [](const Rows& r) { return (reinterpret_cast<uintptr_t>(r.p) & 15u) == 0 && r.slot % 4 == 0 && r.token % 4 == 0 && r.head % 4 == 0; };
    const Rows out = { a.out, a.out_slot, a.out_token, a.out_head };
    if (a.d % 4 == 0 && aligned(a.q) && aligned(a.k) && aligned(a.v) && aligned(out)) hipLaunchKernelGGL((block_attn_f32_kernel<DQ, true>), dim3((unsigned)items), dim3(kF32Waves * 64), 0, st, a, q_tiles);
    else hipLaunchKernelGGL((block_attn_f32_kernel<DQ, false>), dim3((unsigned)items), dim3(kF32Waves * 64), 0, st, a, q_tiles);
    DRF_HIP(hipGetLastError());
    return DRF_OK;
}

drf_status launch_block_attn(const BlockArgs& a, drf_dtype dtype, hipStream_t st)
{
    if (dtype == DRF_F32) {
        switch ((a.d + 15) / 16) {
        case 1: return launch_f32<1>(a, st);
        case 2: return launch_f32<2>(a, st);
        case 3: case 4: return launch_f32<4>(a, st);
        case 5: case 6: return launch_f32<6>(a, st);
        default: return launch_f32<8>(a, st);
        }
    }
    switch (a.d / 8) {
    case 1: return launch_bf16<1>(a, st);
    case 2: return launch_bf16<2>(a, st);
    case 3: return launch_bf16<3>(a, st);
    case 4: return launch_bf16<4>(a, st);
    case 5: return launch_bf16<5>(a, st);
    case 6: return launch_bf16<6>(a, st);
    case 7: return launch_bf16<7>(a, st);
    case 8: return launch_bf16<8>(a, st);
    case 9: return launch_bf16<9>(a, st);
    case 10: return launch_bf16<10>(a, st);
    case 11: return launch_bf16<11>(a, st);
    case 12: return launch_bf16<12>(a, st);
    case 13: return launch_bf16<13>(a, st);
    case 14: return launch_bf16<14>(a, st);
    case 15: return launch_bf16<15>(a, st);
    default: return launch_bf16<16>(a, st);
    }
}

}  // namespace

}  // namespace drf

using namespace drf;

extern "C" size_t drf_block_attention_scratch_bytes(const drf_attn_shape* shape)
{
    if (!shape || shape->slots < 0 || shape->q_tokens < 0 || shape->kv_tokens < 0 || shape->q_heads < 1 || shape->head_dim < 1 || shape->head_dim > kMaxD) return 0;
    return parts_bytes(*shape, split_of(*shape));
}

extern "C" drf_status drf_block_attention(const drf_attn_shape* shape, int q_block, int kv_block, float scale, const uint32_t* blocks,
                                          const drf_heads* q, const drf_heads* k, const drf_heads* v, const drf_heads* out, void* hip_stream)
{
    return drf_block_attention_split(shape, q_block, kv_block, scale, blocks, q, k, v, out, nullptr, 0, hip_stream);
}

extern "C" drf_status drf_block_attention_split(const drf_attn_shape* shape, int q_block, int kv_block, float scale, const uint32_t* blocks,
                                                const drf_heads* q, const drf_heads* k, const drf_heads* v, const drf_heads* out, void* scratch,
                                                size_t scratch_bytes, void* hip_stream)
{
    if (!shape) DRF_FAIL(DRF_EINVAL, "shape is NULL");
    const drf_attn_shape& s = *shape;
    if (s.dtype != DRF_F32 && s.dtype != DRF_BF16) DRF_FAIL(DRF_EINVAL, "unknown dtype");
    if (s.slots < 0 || s.q_tokens < 0 || s.kv_tokens < 0 || s.q_heads < 1 || s.kv_heads < 1 || s.head_dim < 1)
        DRF_FAIL(DRF_EINVAL, "slots and tokens must be >= 0, heads and head_dim >= 1");
    if (s.q_heads % s.kv_heads) DRF_FAIL(DRF_ESHAPE, "%d query heads are no multiple of %d kv heads", s.q_heads, s.kv_heads);
    if (s.head_dim > kMaxD) DRF_FAIL(DRF_ESHAPE, "head_dim must be <= %d (got %d)", kMaxD, s.head_dim);
    if (!log2_of(q_block) || !log2_of(kv_block)) DRF_FAIL(DRF_EINVAL, "blocks of %d queries and %d keys: each must be 32, 64 or 128", q_block, kv_block);
    if (!(scale > 0.f) || !std::isfinite(1.4426950408889634f * scale)) DRF_FAIL(DRF_EINVAL, "scale must be a positive number (and below 2.3e38)");
    if (s.q_tokens > 1 << 30 || s.kv_tokens > 1 << 30) DRF_FAIL(DRF_ESHAPE, "more than 2^30 tokens");
    if (s.slots == 0 || s.q_tokens == 0) return DRF_OK;
    if (!q || !k || !v || !out || !q->data || !out->data || (s.kv_tokens > 0 && (!k->data || !v->data || !blocks))) DRF_FAIL(DRF_EINVAL, "NULL buffer");
    const drf_heads tq = used_strides(*q, s.slots, s.q_tokens, s.q_heads), to = used_strides(*out, s.slots, s.q_tokens, s.q_heads);
    const drf_heads tk = used_strides(*k, s.slots, s.kv_tokens, s.kv_heads), tv = used_strides(*v, s.slots, s.kv_tokens, s.kv_heads);
    for (const drf_heads& t : { tq, tk, tv, to }) {
        if (s.dtype == DRF_BF16 && ((reinterpret_cast<uintptr_t>(t.data) & 15u) || t.slot_stride % 8 || t.token_stride % 8 || t.head_stride % 8))
            DRF_FAIL(DRF_ESHAPE, "bf16 needs 16-byte aligned tensors with strides %% 8 == 0");
        if (t.token_stride < 0 || t.token_stride >= 1 << 24) DRF_FAIL(DRF_ESHAPE, "token stride %lld outside [0, 2^24)", (long long)t.token_stride);
    }
    if (rows_overlap(to, s.slots, s.q_tokens, s.q_heads, s.head_dim)) DRF_FAIL(DRF_EINVAL, "rows of the output lie on one another");
    if (s.dtype == DRF_BF16 && s.head_dim % 8) DRF_FAIL(DRF_ESHAPE, "bf16 needs head_dim %% 8 == 0 (got %d)", s.head_dim);
    BlockArgs a{};
    a.q = { tq.data, tq.slot_stride, tq.token_stride, tq.head_stride };
    a.k = { tk.data, tk.slot_stride, tk.token_stride, tk.head_stride };
    a.v = { tv.data, tv.slot_stride, tv.token_stride, tv.head_stride };
    a.out = to.data; a.out_slot = to.slot_stride; a.out_token = to.token_stride; a.out_head = to.head_stride;
    a.blocks = blocks; a.q_lens = s.q_lens; a.kv_lens = s.kv_lens;
    a.slots = s.slots; a.nq = s.q_tokens; a.nk = s.kv_tokens; a.q_heads = s.q_heads; a.group = s.q_heads / s.kv_heads; a.d = s.head_dim;
    a.q_shift = log2_of(q_block); a.kv_shift = log2_of(kv_block);
    a.q_blocks = (int)(((long long)s.q_tokens + q_block - 1) / q_block);
    a.words = (int)drf_block_words(s.kv_tokens, kv_block);
    a.scale_log2 = 1.4426950408889634f * scale;
    a.split = 1;
    const int split = scratch ? split_of(s) : 1;
    if (split > 1) {
        if (reinterpret_cast<uintptr_t>(scratch) & 15u) DRF_FAIL(DRF_EINVAL, "scratch must be 16-byte aligned");
        if (scratch_bytes < parts_bytes(s, split)) DRF_FAIL(DRF_EINVAL, "scratch of %zu bytes, %zu are needed", scratch_bytes, parts_bytes(s, split));
        a.split = split;
        a.parts = (float*)scratch;
    }
    return launch_block_attn(a, s.dtype, (hipStream_t)hip_stream);
}
