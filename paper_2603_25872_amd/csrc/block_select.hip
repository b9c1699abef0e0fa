// The key blocks that each block of queries attends to: means of the rows of every block in double precision, their products, and the topk
// largest of each row of products.
//
// Which blocks are chosen must not depend on the order of a sum, so nothing before the comparison is narrower than 64 bits (a sum of
// bf16 rows is then exact unless their exponents lie 37 apart), and equal scores go to the lower block.  Sums are divided by their rows before the
// product, not after it: blocks of equal rows then have equal means and equal scores, however many rows the last of them holds.
// The first launch reads q and k once and is bound by that; the means, 1 / block of it, stay in the L2s for the second.
#include <type_traits>

#include "common.h"

namespace drf {

namespace {

typedef double f64x4 __attribute__((ext_vector_type(4)));
typedef double f64x2 __attribute__((ext_vector_type(2)));

constexpr int kMaxD = 128, kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxBlocks = 1024;            // key blocks: 16 rows of scores fill 128 of a CU's 160 KB of LDS

struct PoolSide {
    const void* x;
    int64_t xs, xt, xh;
    int tokens, heads, block, blocks;
    const int32_t* lens;
    double* out;        // means [slot][head][blocks up to a multiple of 16][columns up to a multiple of 8]
};

// A wave takes a head of a block: 64 / P rows at a time in pieces of 16 bytes (VEC), or a row at a time, a column or two a lane.  Bound by the read
// of q and k: 64 slots x 1024 tokens x 32 heads of 72 in bf16, 302 MB, 63 us (4.8 TB/s); 2 x 19344 x 16 heads of 64 in fp32, 158 MB, 39 us
// (4.0) from memory and 16 out of the Infinity Cache.  Six rows in flight a lane, and a block's means stored as one row: by columns, where 8 bytes of a line leave at a time, the first took 87 us.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) pool_kernel(const PoolSide q, const PoolSide k, int d, int q_groups, int parts)
{
    constexpr int E = VEC ? 16 / (int)sizeof(T) : 2;
    typedef T piece __attribute__((ext_vector_type(16 / sizeof(T))));
    __shared__ double part_sums[kWaves][64 * (16 / sizeof(T))];
    int id = blockIdx.x;
    const bool is_k = id >= q_groups;
    const PoolSide& s = is_k ? k : q;
    if (is_k) id -= q_groups;
    const int part = id % parts;
    id /= parts;
    const int slot = id / s.blocks, block = id - slot * s.blocks, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int len = slot_len(s.lens, slot, s.tokens), n0 = block * s.block, end = n0 + s.block < len ? n0 + s.block : len;
    const int width = (d + 7) / 8 * 8, padded = (s.blocks + 15) / 16 * 16;
    const double rows = end > n0 ? end - n0 : 1;                // (of a block behind the length the mean is zero, and not compared)
    for (int h = part * kWaves + wave; h < s.heads; h += parts * kWaves) {
        const T* x = (const T*)s.x + slot * s.xs + h * s.xh;
        double* out = s.out + (((size_t)slot * s.heads + h) * padded + block) * width;
        double sum[E];
#pragma unroll
        for (int j = 0; j < E; ++j) sum[j] = 0.0;
        if constexpr (VEC) {
            const int P = d / E, rpw = 64 / P, lr = lane / P, lp = lane - lr * P;
            constexpr int U = 6;                                // rows in flight
            for (int n = n0 + lr; n < end && lr < rpw; n += U * rpw) {
                piece v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const piece*>(x + (int64_t)(n + u * rpw < end ? n + u * rpw : n) * s.xt + lp * E);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (n + u * rpw < end) {
#pragma unroll
                        for (int j = 0; j < E; ++j) sum[j] += (double)(float)v[u][j];
                    }
            }
            double* mine = part_sums[wave];                     // (a wave's LDS operations complete in order)
#pragma unroll
            for (int j = 0; j < E; ++j) mine[lane * E + j] = sum[j];
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            for (int c = lane; c < width; c += 64) {
                double t = 0.0;
                if (c < d)
                    for (int r = 0; r < rpw; ++r) t += mine[r * d + c];
                out[c] = t / rows;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        } else {
            for (int n = n0; n < end; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (lane + 64 * j < d) sum[j] += (double)(float)x[(int64_t)n * s.xt + lane + 64 * j];
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if (lane + 64 * j < width) out[lane + 64 * j] = sum[j] / rows;
        }
    }
}

// Unsigned keys in the order of the scores, none of them 0; one that is not a number below all.
__device__ inline uint64_t key_of(double v)
{
    if (v != v) return 1;
    v += 0.0;                                                   // -0 and 0 are equal
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

struct SelectArgs {
    const double *q, *k;
    int q_tokens, kv_tokens, q_heads, group, q_block, kv_block, nq, nk, pairs, topk, words;      // pairs: of k-steps, 8 columns each
    const int32_t *q_lens, *kv_lens;
    uint32_t* blocks;
};

// A workgroup takes 16 query blocks of a (slot, head): their scores against all key blocks on the 16 x 16 x 4 matrix instruction into LDS, then a
// wave row after row.  Up to 64 blocks a row (NK = 1, a key a lane) every key's rank is counted against one key after another, four
// instructions each; more of them have the topk-th largest key found by bisection over its bits, the upper 32 first, on scalars but for the
// comparisons (counting by ballots, until a bound splits off exactly topk).  Latency bounds both, and with many rows of few blocks the instructions:
// 2 slots x 8 heads x 152 rows of 303 blocks 16 us on 160 workgroups (21.9 with two batches of sums a tile and 64-bit comparisons throughout; 4 of
// it are the bisection), 64 x 16 x 16 rows of 16 blocks 11.  Nine pairs at once are slower where eight do (17.0).  NK: keys of a row that a lane
// holds; NW: waves.
constexpr int kRows = 16;
template <int NK, int NW>
__global__ void __launch_bounds__(NW * 64) select_kernel(const SelectArgs a)
{
    constexpr int R = kRows / NW, kPairs = NW == 16 ? 8 : 6;                // pairs of k-steps asked for at once
    extern __shared__ __attribute__((aligned(16))) double score[];          // [16][nk padded]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int qtiles = (a.nq + 15) / 16, ktiles = (a.nk + 15) / 16, ld = ktiles * 16 + 2;
    // the rows of one head on one XCD: they read the same means of keys
    const int id = item_by_xcd(blockIdx.x, gridDim.x);
    const int qt = id % qtiles, sh = id / qtiles, slot = sh / a.q_heads, h = sh - slot * a.q_heads;
    const int q_len = slot_len(a.q_lens, slot, a.q_tokens), kv_len = slot_len(a.kv_lens, slot, a.kv_tokens);
    const int n_valid = (kv_len + a.kv_block - 1) / a.kv_block;             // key blocks that hold a key
    // Operands of the product: row lane % 16 of a tile, and of every 8 columns 2 (lane / 16) in one k-step, the next in another (16 bytes a lane).
    const int width = 8 * a.pairs;
    const double* q = a.q + (((size_t)sh * qtiles + qt) * 16 + (lane & 15)) * width + 2 * (lane >> 4);
    const double* k = a.k + (((size_t)slot * (a.q_heads / a.group) + h / a.group) * ktiles * 16 + (lane & 15)) * width + 2 * (lane >> 4);
    f64x2 qv[kPairs];                                                       // stay where they are all of a row's
    for (int t = wave; t < ktiles; t += NW) {
        const double* kt = k + (size_t)t * 16 * width;
        f64x4 acc[2] = { { 0.0, 0.0, 0.0, 0.0 }, { 0.0, 0.0, 0.0, 0.0 } };
        for (int s0 = 0; s0 < a.pairs; s0 += kPairs) {
            f64x2 kv[kPairs];
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                const int s = s0 + j < a.pairs ? s0 + j : a.pairs - 1;
                if (t == wave || a.pairs > kPairs) qv[j] = *reinterpret_cast<const f64x2*>(q + s * 8);
                kv[j] = *reinterpret_cast<const f64x2*>(kt + s * 8);
            }
#pragma unroll
            for (int j = 0; j < kPairs; ++j)
                if (s0 + j < a.pairs) {
                    acc[0] = __builtin_amdgcn_mfma_f64_16x16x4f64(qv[j][0], kv[j][0], acc[0], 0, 0, 0);
                    acc[1] = __builtin_amdgcn_mfma_f64_16x16x4f64(qv[j][1], kv[j][1], acc[1], 0, 0, 0);
                }
        }
        // lane l holds column l % 16 of rows l / 16 + 4 r
#pragma unroll
        for (int r = 0; r < 4; ++r) score[((lane >> 4) + 4 * r) * ld + t * 16 + (lane & 15)] = acc[0][r] + acc[1][r];
    }
    __syncthreads();
    for (int r = 0; r < R; ++r) {
        const int i = qt * kRows + wave * R + r;
        if (i >= a.nq) break;
        const int want = i * a.q_block >= q_len ? 0 : a.topk < n_valid ? a.topk : n_valid;
        uint64_t key[NK], chosen[NK];
#pragma unroll
        for (int c = 0; c < NK; ++c) key[c] = c * 64 + lane < n_valid ? key_of(score[(wave * R + r) * ld + c * 64 + lane]) : 0;
        uint64_t least = 0;                                                 // the want-th largest key, or what splits as many off
        int above = want > 0 ? n_valid : 0;                                 // keys >= least
        if (want > 0 && want < n_valid) {
            if constexpr (NK == 1) {
                int rank = 0;                                               // keys above this lane's
                for (int j = 0; j < n_valid; ++j) {
                    const uint64_t other = (uint64_t)__builtin_amdgcn_readlane((uint32_t)(key[0] >> 32), j) << 32 | (uint32_t)__builtin_amdgcn_readlane((uint32_t)key[0], j);
                    rank += other > key[0];
                }
                // those with fewer than `want` above them: as many, or more if the least of them come several times
                const uint64_t in = __ballot(key[0] != 0 && rank < want);
                above = __popcll(in);
                least = 1;
                if (above == want) {
                    key[0] = in >> lane & 1;                                // (1: chosen)
                } else {
                    int most = in >> lane & 1 ? rank : -1;
#pragma unroll
                    for (int o = 32; o; o >>= 1) { const int u = __shfl_xor(most, o, 64); most = u > most ? u : most; }
                    const int at = __builtin_ctzll(__ballot((in >> lane & 1) && rank == most));
                    least = (uint64_t)__builtin_amdgcn_readlane((uint32_t)(key[0] >> 32), at) << 32 | (uint32_t)__builtin_amdgcn_readlane((uint32_t)key[0], at);
                }
            } else {
                uint32_t high[NK], low = 0;
#pragma unroll
                for (int c = 0; c < NK; ++c) high[c] = (uint32_t)(key[c] >> 32);
                for (int b = 31; b >= 0 && above != want; --b) {
                    const uint32_t bound = low | 1u << b;
                    int n = 0;
#pragma unroll
                    for (int c = 0; c < NK; ++c) n += __popcll(__ballot(high[c] >= bound));
                    if (n >= want) { low = bound; above = n; }
                }
                least = (uint64_t)low << 32;
                for (int b = 31; b >= 0 && above != want; --b) {
                    const uint64_t bound = least | 1ull << b;
                    int n = 0;
#pragma unroll
                    for (int c = 0; c < NK; ++c) n += __popcll(__ballot(key[c] >= bound));
                    if (n >= want) { least = bound; above = n; }
                }
            }
        }
#pragma unroll
        for (int c = 0; c < NK; ++c) chosen[c] = above ? __ballot(key[c] != 0 && key[c] >= least) : 0;
        if (above != want) {
            // of the keys equal to the least as many too many: the last of them go
            int more = 0;
#pragma unroll
            for (int c = 0; c < NK; ++c) more += __popcll(__ballot(key[c] > least));
            int equal = want - more;
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                const uint64_t same = __ballot(key[c] == least);
                const int before = __popcll(same & ((1ull << lane) - 1)), here = __popcll(same);
                chosen[c] = __ballot(key[c] > least || (key[c] == least && before < equal));
                equal = equal > here ? equal - here : 0;
            }
        }
        uint32_t* out = a.blocks + ((size_t)sh * a.nq + i) * a.words;
#pragma unroll
        for (int c = 0; c < NK; ++c)
            if (lane < 2 && 2 * c + lane < a.words) out[2 * c + lane] = (uint32_t)(chosen[c] >> (32 * lane));
    }
}

bool block_size(int b) { return b == 32 || b == 64 || b == 128; }

drf_status check_select(const drf_attn_shape* s, int q_block, int kv_block)
{
    if (!s) DRF_FAIL(DRF_EINVAL, "shape is NULL");
    if (s->dtype != DRF_F32 && s->dtype != DRF_BF16) DRF_FAIL(DRF_EINVAL, "unknown dtype");
    if (s->slots < 0 || s->q_tokens < 0 || s->kv_tokens < 0 || s->q_heads < 1 || s->kv_heads < 1 || s->head_dim < 1)
        DRF_FAIL(DRF_EINVAL, "slots and tokens must be >= 0, heads and head_dim >= 1");
    if (s->q_heads % s->kv_heads) DRF_FAIL(DRF_ESHAPE, "%d query heads are no multiple of %d kv heads", s->q_heads, s->kv_heads);
    if (s->head_dim > kMaxD) DRF_FAIL(DRF_ESHAPE, "head_dim must be <= %d (got %d)", kMaxD, s->head_dim);
    if (!block_size(q_block) || !block_size(kv_block)) DRF_FAIL(DRF_EINVAL, "blocks of %d queries and %d keys: each must be 32, 64 or 128", q_block, kv_block);
    return DRF_OK;
}

size_t side_bytes(int slots, int heads, int blocks, int d)
{
    return (size_t)slots * heads * ((blocks + 15) / 16 * 16) * ((d + 7) / 8 * 8) * sizeof(double);
}

template <int NK, int NW> drf_status launch_select(const SelectArgs& a, unsigned grid, size_t lds, hipStream_t st)
{
    auto kern = select_kernel<NK, NW>;
    static std::atomic<uint64_t> lds_allowed{ 0 };
    DRF_HIP(allow_lds(reinterpret_cast<const void*>(kern), kRows * (64 * NK + 2) * (int)sizeof(double), lds_allowed));
    hipLaunchKernelGGL(kern, dim3(grid), dim3(NW * 64), lds, st, a);
    DRF_HIP(hipGetLastError());
    return DRF_OK;
}

}  // namespace

}  // namespace drf

using namespace drf;

extern "C" size_t drf_block_words(int kv_tokens, int kv_block)
{
    if (kv_tokens < 0 || !block_size(kv_block)) return 0;
    const long long blocks = ((long long)kv_tokens + kv_block - 1) / kv_block;
    return (size_t)((blocks + 31) / 32);
}

extern "C" size_t drf_block_select_scratch_bytes(const drf_attn_shape* shape, int q_block, int kv_block)
{
    if (check_select(shape, q_block, kv_block) != DRF_OK) return 0;
    const int nq = (int)(((long long)shape->q_tokens + q_block - 1) / q_block), nk = (int)(((long long)shape->kv_tokens + kv_block - 1) / kv_block);
    return side_bytes(shape->slots, shape->q_heads, nq, shape->head_dim) + side_bytes(shape->slots, shape->kv_heads, nk, shape->head_dim);
}

extern "C" drf_status drf_block_select(const drf_attn_shape* shape, int q_block, int kv_block, int topk, const drf_heads* q,
                                       const drf_heads* k, void* scratch, size_t scratch_bytes, uint32_t* blocks, void* hip_stream)
{
    drf_status rc = check_select(shape, q_block, kv_block);
    if (rc != DRF_OK) return rc;
    const drf_attn_shape& s = *shape;
    if (topk < 1) DRF_FAIL(DRF_EINVAL, "topk must be >= 1 (got %d)", topk);
    const int nq = (int)(((long long)s.q_tokens + q_block - 1) / q_block), nk = (int)(((long long)s.kv_tokens + kv_block - 1) / kv_block);
    if (nk > kMaxBlocks) DRF_FAIL(DRF_ESHAPE, "%d key blocks exceed the %d that are compared", nk, kMaxBlocks);
    if (s.slots == 0 || s.q_tokens == 0 || s.kv_tokens == 0) return DRF_OK;         // no row, or rows of no words
    if (!q || !k || !q->data || !k->data || !blocks || !scratch) DRF_FAIL(DRF_EINVAL, "NULL buffer");
    if ((reinterpret_cast<uintptr_t>(scratch) & 15u) != 0) DRF_FAIL(DRF_EINVAL, "scratch must be 16-byte aligned");
    const size_t q_bytes = side_bytes(s.slots, s.q_heads, nq, s.head_dim), need = q_bytes + side_bytes(s.slots, s.kv_heads, nk, s.head_dim);
    if (scratch_bytes < need) DRF_FAIL(DRF_EINVAL, "scratch of %zu bytes, %zu are needed", scratch_bytes, need);
    hipStream_t st = (hipStream_t)hip_stream;

    const int unit = s.dtype == DRF_BF16 ? 8 : 4;
    bool vec = s.head_dim % unit == 0;
    auto side = [&](const drf_heads* x, int tokens, int heads, int block, int n, const int32_t* lens, double* out) {
        const drf_heads t = used_strides(*x, s.slots, tokens, heads);
        vec = vec && (reinterpret_cast<uintptr_t>(t.data) & 15u) == 0 && t.slot_stride % unit == 0 && t.token_stride % unit == 0 && t.head_stride % unit == 0;
        return PoolSide{ t.data, t.slot_stride, t.token_stride, t.head_stride, tokens, heads, block, n, lens, out };
    };
    double* q_means = (double*)scratch;
    double* k_means = (double*)((char*)scratch + q_bytes);
    const PoolSide qs = side(q, s.q_tokens, s.q_heads, q_block, nq, s.q_lens, q_means), ks = side(k, s.kv_tokens, s.kv_heads, kv_block, nk, s.kv_lens, k_means);
    int parts = 1;                                                          // workgroups over the heads of a block
    while (parts * kWaves < s.q_heads && (long long)s.slots * (nq + nk) * parts < 2048) parts *= 2;
    const long long q_groups = (long long)s.slots * nq * parts, groups = q_groups + (long long)s.slots * nk * parts;
    const long long rows = (long long)s.slots * s.q_heads * ((nq + 15) / 16);
    if (groups > 0x7fffffLL || rows > 0x1fffffLL) DRF_FAIL(DRF_ESHAPE, "too many blocks");
    auto pool = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(kThreads), 0, st, qs, ks, s.head_dim, (int)q_groups, parts); };
    if (s.dtype == DRF_BF16) vec ? pool(pool_kernel<bf16_t, true>) : pool(pool_kernel<bf16_t, false>);
    else vec ? pool(pool_kernel<float, true>) : pool(pool_kernel<float, false>);
    DRF_HIP(hipGetLastError());

    SelectArgs a{};
    a.q = q_means; a.k = k_means; a.q_tokens = s.q_tokens; a.kv_tokens = s.kv_tokens; a.q_heads = s.q_heads; a.group = s.q_heads / s.kv_heads;
    a.q_block = q_block; a.kv_block = kv_block; a.nq = nq; a.nk = nk; a.pairs = (s.head_dim + 7) / 8; a.topk = topk;
    a.words = (int)drf_block_words(s.kv_tokens, kv_block); a.q_lens = s.q_lens; a.kv_lens = s.kv_lens; a.blocks = blocks;
    const size_t lds = (size_t)kRows * ((nk + 15) / 16 * 16 + 2) * sizeof(double);
    if (nk <= 64) return launch_select<1, 4>(a, (unsigned)rows, lds, st);
    if (nk <= 128) return launch_select<2, 16>(a, (unsigned)rows, lds, st);
    if (nk <= 256) return launch_select<4, 16>(a, (unsigned)rows, lds, st);
    if (nk <= 512) return launch_select<8, 16>(a, (unsigned)rows, lds, st);
    return launch_select<16, 16>(a, (unsigned)rows, lds, st);
}
