// Attention over the key blocks that a bit mask gives each block of queries.
//
// bf16: flash-style, a wave takes 32 queries of one query block and walks its list of key blocks in steps of 32 keys.  Scores are computed
// transposed (S^T = K Q^T), so that a lane owns one query column: the online softmax needs one exchange between the halves of a wave, and the
// probabilities are where the second product (O^T = V^T P^T) wants them.  A block that is not chosen is never read.
// fp32: a workgroup takes 16 queries, its four waves the steps in turn, each with a softmax of its own; joined through LDS.
#include <type_traits>

#include "common.h"

namespace drf {

namespace {

typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
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
};

__device__ inline int slot_len(const int32_t* lens, int slot, int tokens)
{
    if (!lens) return tokens;
    const int n = lens[slot];
    return n < 0 ? 0 : n < tokens ? n : tokens;
}

// The steps of 32 keys of a query block's list, every `stride`-th of them from number `first` on.
struct Walk {
    const uint32_t* row; int words, len, shift, stride, skip;
    int w = -1, block = 0, sub = 0, subs = 0; uint32_t bits = 0;
    __device__ Walk(const BlockArgs& a, int slot, int h, int q0, int len_, int first, int stride_)
        : row(a.blocks + (((size_t)slot * a.q_heads + h) * a.q_blocks + (q0 >> a.q_shift)) * a.words), words(a.words), len(len_), shift(a.kv_shift),
          stride(stride_), skip(first) {}
    // first key of the next step; -1: none
    __device__ int next()
    {
        for (;;) {
            if (sub == subs) {
                while (bits == 0) {
                    if (++w >= words) { w = words; return -1; }
                    bits = __builtin_amdgcn_readfirstlane(row[w]);
                }
                block = 32 * w + __builtin_ctz(bits);
                bits &= bits - 1;
                const int left = len - (block << shift);
                sub = 0;
                subs = left <= 0 ? 0 : left >= 1 << shift ? 1 << (shift - 5) : (left + kStep - 1) / kStep;
                if (subs == 0) continue;
            }
            const int kv0 = (block << shift) + kStep * sub++;
            if (skip-- == 0) { skip = stride - 1; return kv0; }
        }
    }
};

template <int P8>
__global__ void __launch_bounds__(64) block_attn_kernel(const BlockArgs a, int q_tiles)
{
    constexpr int d = P8 * 8, KS = (P8 + 1) / 2, DT = (d + 31) / 32, DK = KS * 16;
    constexpr int LDK = DK + 8, LDV = DT * 32 + 16, LDO = DT * 32 + 8, PIECES = kStep * P8 / 64 + (kStep * P8 % 64 != 0);
    __shared__ __attribute__((aligned(16))) bf16_t sK[kStep * LDK], sV[kStep * LDV], sO[32 * LDO];
    const int lane = threadIdx.x, l32 = lane & 31, half = lane >> 5;
    const int tile = blockIdx.x % q_tiles, sh = blockIdx.x / q_tiles, slot = sh / a.q_heads, h = sh - slot * a.q_heads;
    const int q0 = tile * 32, q_len = slot_len(a.q_lens, slot, a.nq), kv_len = slot_len(a.kv_lens, slot, a.nk);
    if (q0 >= q_len) return;
    const bf16x8 zero8 = { 0, 0, 0, 0, 0, 0, 0, 0 };
    const bf16_t* Q = (const bf16_t*)a.q.p + slot * a.q.slot + h * a.q.head;
    const bf16_t* K = (const bf16_t*)a.k.p + slot * a.k.slot + h / a.group * a.k.head;
    const bf16_t* V = (const bf16_t*)a.v.p + slot * a.v.slot + h / a.group * a.v.head;
    bf16x8 qf[KS];
    {
        const int q = q0 + l32 < q_len ? q0 + l32 : q_len - 1;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int c = ks * 16 + half * 8;
            qf[ks] = c < d ? *reinterpret_cast<const bf16x8*>(Q + (int64_t)q * a.q.token + c) : zero8;
        }
    }
    for (int i = lane; i < kStep * LDK / 8; i += 64) reinterpret_cast<bf16x8*>(sK)[i] = zero8;
    for (int i = lane; i < kStep * LDV / 8; i += 64) reinterpret_cast<bf16x8*>(sV)[i] = zero8;
    f32x16 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    Walk walk(a, slot, h, q0, kv_len, 0, 1);
    __syncthreads();
    for (int kv0 = walk.next(); kv0 >= 0; kv0 = walk.next()) {
        const int left = kv_len - kv0;
        bf16x8 rk[PIECES], rv[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int id = lane + 64 * i, r = id / P8, c = id % P8;
            rk[i] = rv[i] = zero8;                              // rows behind the last key: their scores are masked, their values zero
            if (id < kStep * P8 && r < left) {
                rk[i] = *reinterpret_cast<const bf16x8*>(K + (int64_t)(kv0 + r) * a.k.token + c * 8);
                rv[i] = *reinterpret_cast<const bf16x8*>(V + (int64_t)(kv0 + r) * a.v.token + c * 8);
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int id = lane + 64 * i, r = id / P8, c = id % P8;
            if (id < kStep * P8) {
                *reinterpret_cast<bf16x8*>(sK + r * LDK + c * 8) = rk[i];
                *reinterpret_cast<bf16x8*>(sV + r * LDV + c * 8) = rv[i];
            }
        }
        __syncthreads();
        f32x16 s = { 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f };
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(sK + l32 * LDK + ks * 16 + half * 8), qf[ks], s, 0, 0, 0);
        // register r holds key 8 (r / 4) + 4 half + r % 4 of the step
        float mx = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if (8 * (r >> 2) + 4 * half + (r & 3) >= left) s[r] = -INFINITY;
            mx = fmaxf(mx, s[r]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m_run, mx);
        const float ref = m_new == -INFINITY ? 0.f : m_new;     // nothing above -infinity yet: numerators are zero against any
        const float alpha = __builtin_amdgcn_exp2f((m_run - ref) * a.scale_log2);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[t][r] *= alpha;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f((s[r] - ref) * a.scale_log2);
            l_run += s[r];
        }
        // V^T operand by the transposing LDS read: lane i of 16 receives column i of 4 rows, rows 16 c + 4 half + 0..3 and the same + 8
        const bf16_t* vl = sV + (4 * half + ((lane & 15) >> 2)) * LDV + (l32 & 16) + 4 * (lane & 3);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            bf16x8 pf;
#pragma unroll
            for (int e = 0; e < 8; ++e) pf[e] = (bf16_t)s[8 * c + e];
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((DRF_LDS_PTR s16x4*)(vl + 16 * c * LDV + t * 32));
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((DRF_LDS_PTR s16x4*)(vl + (16 * c + 8) * LDV + t * 32));
                o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)), pf, o[t], 0, 0, 0);
            }
        }
    }
    const float l_tot = l_run + __shfl_xor(l_run, 32, 64), inv = l_tot > 0.f ? 1.f / l_tot : l_tot != l_tot ? l_tot : 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const bf16x4 w = { (bf16_t)(o[t][4 * g] * inv), (bf16_t)(o[t][4 * g + 1] * inv), (bf16_t)(o[t][4 * g + 2] * inv), (bf16_t)(o[t][4 * g + 3] * inv) };
            *reinterpret_cast<bf16x4*>(sO + l32 * LDO + t * 32 + 8 * g + 4 * half) = w;
        }
    __syncthreads();
    bf16_t* op = (bf16_t*)a.out + slot * a.out_slot + h * a.out_head;
    for (int id = lane; id < 32 * P8; id += 64) {
        const int r = id / P8, c = id % P8;
        if (q0 + r < q_len) *reinterpret_cast<bf16x8*>(op + (int64_t)(q0 + r) * a.out_token + c * 8) = *reinterpret_cast<const bf16x8*>(sO + r * LDO + c * 8);
    }
}

// fp32 on the fp32 matrix instruction (16 x 16 x 4), operands straight from memory; DQ = ceil(d / 16).
constexpr int kF32Waves = 4;
template <int DQ>
__global__ void __launch_bounds__(kF32Waves * 64) block_attn_f32_kernel(const BlockArgs a, int q_tiles)
{
    __shared__ f32x4 po[kF32Waves][DQ][64];
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
    f32x4 qf[DQ], o[DQ];
#pragma unroll
    for (int c = 0; c < DQ; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int col = c * 16 + 4 * quarter + j;
            qf[c][j] = col < d ? Q[col] : 0.f;
            o[c][j] = 0.f;
        }
    float m_run = -INFINITY, l_run = 0.f;                       // l_run: this quarter's share
    Walk walk(a, slot, h, q0, kv_len, wave, kF32Waves);
    for (int kv0 = walk.next(); kv0 >= 0; kv0 = walk.next()) {
        f32x4 s[2];
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int row = kv0 + 16 * t + l16, rc = row < kv_len ? row : kv_len - 1;
            const float* kr = K + (int64_t)rc * a.k.token;
            s[t] = (f32x4){ 0.f, 0.f, 0.f, 0.f };
#pragma unroll
            for (int c = 0; c < DQ; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int col = c * 16 + 4 * quarter + j;
                    s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(col < d ? kr[col] : 0.f, qf[c][j], s[t], 0, 0, 0);
                }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (kv0 + 16 * t + 4 * quarter + r >= kv_len) s[t][r] = -INFINITY;
                mx = fmaxf(mx, s[t][r]);
            }
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m_run, mx), ref = m_new == -INFINITY ? 0.f : m_new, alpha = exp2f((m_run - ref) * a.scale_log2);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int c = 0; c < DQ; ++c) o[c] *= alpha;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float p = exp2f((s[t][r] - ref) * a.scale_log2);
                l_run += p;
                const int row = kv0 + 16 * t + 4 * quarter + r;
#pragma unroll
                for (int c = 0; c < DQ; ++c) {
                    const float v = row < kv_len && c * 16 + l16 < d ? V[(int64_t)row * a.v.token + c * 16 + l16] : 0.f;
                    o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p, o[c], 0, 0, 0);
                }
            }
    }
    l_run += __shfl_xor(l_run, 16, 64);
    l_run += __shfl_xor(l_run, 32, 64);
    if (quarter == 0) { pm[wave][l16] = m_run; pl[wave][l16] = l_run; }
#pragma unroll
    for (int c = 0; c < DQ; ++c) po[wave][c][lane] = o[c];
    __syncthreads();
    float m_all = pm[0][l16], l_all = 0.f, f[kF32Waves];
#pragma unroll
    for (int w = 1; w < kF32Waves; ++w) m_all = fmaxf(m_all, pm[w][l16]);
#pragma unroll
    for (int w = 0; w < kF32Waves; ++w) {                       // a wave without a score above -infinity has nothing to add
        f[w] = pm[w][l16] == -INFINITY ? 0.f : exp2f((pm[w][l16] - m_all) * a.scale_log2);
        l_all += pl[w][l16] * f[w];
    }
    if (q >= q_len) return;
    const float inv = l_all > 0.f ? 1.f / l_all : l_all != l_all ? l_all : 0.f;
    float* op = (float*)a.out + slot * a.out_slot + (int64_t)q * a.out_token + h * a.out_head;
    for (int c = wave; c < DQ; c += kF32Waves) {
        f32x4 v = po[0][c][lane] * f[0];
#pragma unroll
        for (int w = 1; w < kF32Waves; ++w) v += po[w][c][lane] * f[w];
        v *= inv;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (c * 16 + 4 * quarter + r < d) op[c * 16 + 4 * quarter + r] = v[r];
    }
}

int log2_of(int b) { return b == 32 ? 5 : b == 64 ? 6 : b == 128 ? 7 : 0; }

template <int P8> drf_status launch_bf16(const BlockArgs& a, hipStream_t st)
{
    const int q_tiles = (a.nq + 31) / 32;
    const long long items = (long long)q_tiles * a.q_heads * a.slots;
    if (items > 0x1ffffffLL) DRF_FAIL(DRF_ESHAPE, "too many queries");
    hipLaunchKernelGGL((block_attn_kernel<P8>), dim3((unsigned)items), dim3(64), 0, st, a, q_tiles);
    DRF_HIP(hipGetLastError());
    return DRF_OK;
}

template <int DQ> drf_status launch_f32(const BlockArgs& a, hipStream_t st)
{
    const int q_tiles = (a.nq + 15) / 16;
    const long long items = (long long)q_tiles * a.q_heads * a.slots;
    if (items > 0x7fffffLL) DRF_FAIL(DRF_ESHAPE, "too many queries");
    hipLaunchKernelGGL((block_attn_f32_kernel<DQ>), dim3((unsigned)items), dim3(kF32Waves * 64), 0, st, a, q_tiles);
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

extern "C" drf_status drf_block_attention(const drf_attn_shape* shape, int q_block, int kv_block, float scale, const uint32_t* blocks,
                                          const drf_heads* q, const drf_heads* k, const drf_heads* v, const drf_heads* out, void* hip_stream)
{
    if (!shape) DRF_FAIL(DRF_EINVAL, "shape is NULL");
    const drf_attn_shape& s = *shape;
    if (s.dtype != DRF_F32 && s.dtype != DRF_BF16) DRF_FAIL(DRF_EINVAL, "unknown dtype");
    if (s.slots < 0 || s.q_tokens < 0 || s.kv_tokens < 0 || s.q_heads < 1 || s.kv_heads < 1 || s.head_dim < 1)
        DRF_FAIL(DRF_EINVAL, "slots and tokens must be >= 0, heads and head_dim >= 1");
    if (s.q_heads % s.kv_heads) DRF_FAIL(DRF_ESHAPE, "%d query heads are no multiple of %d kv heads", s.q_heads, s.kv_heads);
    if (s.head_dim > kMaxD) DRF_FAIL(DRF_ESHAPE, "head_dim must be <= %d (got %d)", kMaxD, s.head_dim);
    if (!log2_of(q_block) || !log2_of(kv_block)) DRF_FAIL(DRF_EINVAL, "blocks of %d queries and %d keys: each must be 32, 64 or 128", q_block, kv_block);
    if (!(scale > 0.f) || !std::isfinite(scale)) DRF_FAIL(DRF_EINVAL, "scale must be a positive number");
    if (s.slots == 0 || s.q_tokens == 0) return DRF_OK;
    if (!q || !k || !v || !out || !q->data || !out->data || (s.kv_tokens > 0 && (!k->data || !v->data || !blocks))) DRF_FAIL(DRF_EINVAL, "NULL buffer");
    for (const drf_heads* t : { q, k, v, out }) {
        if (s.dtype == DRF_BF16 && ((reinterpret_cast<uintptr_t>(t->data) & 15u) || t->slot_stride % 8 || t->token_stride % 8 || t->head_stride % 8))
            DRF_FAIL(DRF_ESHAPE, "bf16 needs 16-byte aligned tensors with strides %% 8 == 0");
        if (t->token_stride < 0 || t->token_stride >= 1 << 24) DRF_FAIL(DRF_ESHAPE, "token stride %lld outside [0, 2^24)", (long long)t->token_stride);
    }
    if (s.dtype == DRF_BF16 && s.head_dim % 8) DRF_FAIL(DRF_ESHAPE, "bf16 needs head_dim %% 8 == 0 (got %d)", s.head_dim);
    BlockArgs a{};
    a.q = { q->data, q->slot_stride, q->token_stride, q->head_stride };
    a.k = { k->data, k->slot_stride, k->token_stride, k->head_stride };
    a.v = { v->data, v->slot_stride, v->token_stride, v->head_stride };
    a.out = out->data; a.out_slot = out->slot_stride; a.out_token = out->token_stride; a.out_head = out->head_stride;
    a.blocks = blocks; a.q_lens = s.q_lens; a.kv_lens = s.kv_lens;
    a.slots = s.slots; a.nq = s.q_tokens; a.nk = s.kv_tokens; a.q_heads = s.q_heads; a.group = s.q_heads / s.kv_heads; a.d = s.head_dim;
    a.q_shift = log2_of(q_block); a.kv_shift = log2_of(kv_block);
    a.q_blocks = (int)(((long long)s.q_tokens + q_block - 1) / q_block);
    a.words = (int)drf_block_words(s.kv_tokens, kv_block);
    a.scale_log2 = 1.4426950408889634f * scale;
    return launch_block_attn(a, s.dtype, (hipStream_t)hip_stream);
}
