// Linears of a block that carry more than a product: the gated feed-forward block and a projection with low-rank adapters of many requests.
//
//   feed-forward   u = x [Wg; Wv]^T + b,  p = act(u_g) u_v  in one launch: a tile of the first product takes the rows of Wg and Wv sixteen and sixteen, so that
//                  a lane ends with gate and value of the same columns;  then out = p Wo^T + b
//   adapters       t = s_i x A_i^T  [row][rank] in one launch;  then out = x W^T + t B_i^T + b: the adapter is `rank` more columns of the product's inner
//                  axis, whose operands are a row's t and its own adapter's B
//
// Tiles of 64 rows by 64 rows of the weights on four waves, a wave 32 x 32; 64 bytes of the inner axis a step, staged in LDS through registers a step ahead.
// The weights are the matrix instruction's first operand: a lane ends with four consecutive columns of one row.
#include <algorithm>
#include <type_traits>

#include "gemm_device.h"
#include "rows.h"

namespace drf {

namespace {

enum { LIN_STORE = 0, LIN_GLU = 1, LIN_LOW = 2, LIN_ADAPT = 3 };

struct LinArgs {
    drf_rows x, out;
    const void* w;                      // [N][K], or LIN_LOW: [adapters][N][K]; LIN_GLU: [2 N][K], gates and then values
    const float* bias;                  // [N] (LIN_GLU: [2 N]) or NULL
    const int32_t* lens;
    int slots, tokens, N, K;
    uint32_t tok_magic; int tok_shift;
    int slot_rows;                      // rows that are counted together: tokens (tiles do not cross slots) or slots * tokens
    int tiles_m, tiles_n;               // tiles a counted group of rows; tiles of columns
    long long tiles;
    long long first;                    // tile that this launch begins with
    int act, out_vec, in_vec;
    const int32_t* which;
    const float* scales;
    const float* low;                   // [slots * tokens][rank]
    const void* b;                      // [adapters][N][rank]
    int adapters, rank;
};

template <typename T> struct Step;
template <> struct Step<float> { static constexpr int E = 4; };
template <> struct Step<bf16_t> { static constexpr int E = 8; };

__device__ inline float glu(float a, float v, int act)
{
    if (act == DRF_GLU_GELU) return gelu_tanh(a) * v;
    return a * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * a)) * v;
}

__device__ inline int div_rows(int m, const LinArgs& a) { return fast_div(m, a.tok_magic, a.tok_shift); }

__device__ inline int adapter_of(const LinArgs& a, int slot)
{
    const int i = a.adapters ? a.which[slot] : -1;
    return i >= 0 && i < a.adapters ? i : -1;
}

// c += w . x over 64 bytes of the inner axis, a lane's 16 bytes each
__device__ inline void multiply(f32x4& c, const u32x4& w, const u32x4& x, float)
{
    const f32x4 a = __builtin_bit_cast(f32x4, w), b = __builtin_bit_cast(f32x4, x);
#pragma unroll
    for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[k], b[k], c, 0, 0, 0);
}
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
__device__ inline void multiply(f32x4& c, const u32x4& w, const u32x4& x, bf16_t)
{
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
}

// fp32 values as operands: in bf16 the sum of two, the upper 8 bits and the rest rounded to 8 (2^-16 of the value is lost); one that is no number is itself and zero.
__device__ inline void split(const float (&v)[4], u32x4 (&f)[2], float) { __builtin_memcpy(&f[0], v, 16); }
__device__ inline void split(const float (&v)[8], u32x4 (&f)[2], bf16_t)
{
    bf16_t hi[8], lo[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float top = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v[e]) & 0xffff0000u);
        const bool fine = fabsf(v[e]) < INFINITY;
        hi[e] = (bf16_t)(fine ? top : v[e]);
        lo[e] = (bf16_t)(fine ? v[e] - top : 0.f);
    }
    __builtin_memcpy(&f[0], hi, 16);
    __builtin_memcpy(&f[1], lo, 16);
}

// 16 bytes of a row of n elements from element k on, zeros behind its end
template <typename T> __device__ inline u32x4 load16(const T* row, int k, int n, bool vec)
{
    constexpr int E = Step<T>::E;
    if (vec) return k < n ? *reinterpret_cast<const u32x4*>(row + k) : (u32x4){ 0, 0, 0, 0 };
    T v[E];
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = k + j < n ? row[k + j] : (T)0.f;
    u32x4 r;
    __builtin_memcpy(&r, v, 16);
    return r;
}

template <typename T, int KIND>
__global__ void __launch_bounds__(256) linear_kernel(const LinArgs a)
{
    constexpr int E = Step<T>::E, BK = 4 * E, PITCH = 80;           // bytes of a row of 64 in LDS: 16 rows on distinct banks
    __shared__ __attribute__((aligned(16))) unsigned char stage[2][128 * PITCH];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave & 1, wn = wave >> 1;
    const long long id = a.first + blockIdx.x;
    const int tn = (int)(id % a.tiles_n);
    const long long rest = id / a.tiles_n;
    const int tm = (int)(rest % a.tiles_m), group = (int)(rest / a.tiles_m);
    const int row0 = tm * 64, n0 = tn * (KIND == LIN_GLU ? 32 : 64);
    // row r of the tile: its slot and token; rows that are not there are read as row 0 and not stored
    auto locate = [&](int r, int& slot, int& token) {
        const int m = row0 + r;
        if (a.slot_rows == a.tokens) { slot = group; token = m; }
        else { slot = div_rows(m, a); token = m - slot * a.tokens; }
        return m < a.slot_rows && token < slot_len(a.lens, slot, a.tokens);
    };
    int adapter = -1;
    if constexpr (KIND == LIN_LOW) {
        adapter = adapter_of(a, group);
        if (adapter < 0) return;
    }
    if (a.slot_rows == a.tokens && row0 >= slot_len(a.lens, group, a.tokens)) return;

    // staging: thread t copies the 16-byte pieces t % 4 of rows t / 4 of the activations and of the weights
    const int sr = tid >> 2, sc = (tid & 3) * E;
    int s_slot, s_token;
    if (!locate(sr, s_slot, s_token)) locate(0, s_slot, s_token);
    const T* xr = (const T*)a.x.data + s_slot * a.x.slot_stride + s_token * a.x.token_stride;
    const T* wr = (const T*)a.w;
    if constexpr (KIND == LIN_GLU) {
        int n = n0 + sr / 32 * 16 + sr % 16;
        n = n < a.N ? n : a.N - 1;
        wr += ((size_t)n + (sr / 16 % 2 ? a.N : 0)) * a.K;
    } else {
        int n = n0 + sr;
        n = n < a.N ? n : a.N - 1;
        wr += (KIND == LIN_LOW ? (size_t)adapter * a.N * a.K : 0) + (size_t)n * a.K;
    }
    u32x4 px, pw;
    auto fetch = [&](int k) { px = load16(xr, k + sc, a.K, a.in_vec); pw = load16(wr, k + sc, a.K, a.in_vec); };
    auto put = [&](int s) {
        *reinterpret_cast<u32x4*>(&stage[s][sr * PITCH + (tid & 3) * 16]) = px;
        *reinterpret_cast<u32x4*>(&stage[s][(64 + sr) * PITCH + (tid & 3) * 16]) = pw;
    };
    f32x4 acc[2][2];                                                // [weight piece][activation piece]
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = (f32x4){ 0.f, 0.f, 0.f, 0.f };
    const int steps = (a.K + BK - 1) / BK;
    fetch(0);
    put(0);
    __syncthreads();
    for (int s = 0; s < steps; ++s) {
        if (s + 1 < steps) fetch((s + 1) * BK);
        const unsigned char* st = stage[s & 1];
        u32x4 fx[2], fw[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            fx[i] = *reinterpret_cast<const u32x4*>(st + (wm * 32 + i * 16 + l16) * PITCH + quarter * 16);
            fw[i] = *reinterpret_cast<const u32x4*>(st + (64 + wn * 32 + i * 16 + l16) * PITCH + quarter * 16);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) multiply(acc[i][j], fw[i], fx[j], T{});
        if (s + 1 < steps) put((s + 1) & 1);
        __syncthreads();
    }

    int slot[2], token[2];
    bool live[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        live[j] = locate(wm * 32 + j * 16 + l16, slot[j], token[j]);
        if (!live[j]) slot[j] = token[j] = 0;
    }
    if constexpr (KIND == LIN_ADAPT) {
        int first, last, t;
        locate(0, first, t);
        const int end = std::min(row0 + 64, a.slot_rows) - 1 - row0;
        locate(end, last, t);
        for (int s = first; s <= last; ++s) {                       // (the same for the whole workgroup)
            const int i = adapter_of(a, s);
            if (i < 0) continue;
            const T* b = (const T*)a.b + (size_t)i * a.N * a.rank;
            // into sums of its own, of which the slot's rows take theirs: an infinite weight of one adapter is nothing to the rows of another
            f32x4 sum[2][2];
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int j = 0; j < 2; ++j) sum[p][j] = (f32x4){ 0.f, 0.f, 0.f, 0.f };
            for (int k = 0; k < a.rank; k += BK) {
                u32x4 fw[2], fx[2][2];
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    int n = n0 + wn * 32 + p * 16 + l16;
                    n = n < a.N ? n : a.N - 1;
                    fw[p] = load16(b + (size_t)n * a.rank, k + quarter * E, a.rank, false);
                    float v[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const int c = k + quarter * E + e;
                        v[e] = live[p] && slot[p] == s && c < a.rank ? a.low[((size_t)slot[p] * a.tokens + token[p]) * a.rank + c] : 0.f;
                    }
                    split(v, fx[p], T{});
                }
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        multiply(sum[p][j], fw[p], fx[j][0], T{});
                        if constexpr (sizeof(T) == 2) multiply(sum[p][j], fw[p], fx[j][1], T{});
                    }
            }
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[p][j][r] += slot[j] == s ? sum[p][j][r] : 0.f;
        }
    }

    // acc[i][j][r] is (row 16 j + l16, column 16 i + 4 quarter + r) of the wave's tile
    typedef std::conditional_t<KIND == LIN_LOW, float, T> O;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if (!live[j]) continue;
        O* o = (O*)a.out.data + slot[j] * a.out.slot_stride + token[j] * a.out.token_stride;
#pragma unroll
        for (int i = 0; i < (KIND == LIN_GLU ? 1 : 2); ++i) {
            const int n = n0 + (KIND == LIN_GLU ? wn * 16 : wn * 32 + i * 16) + 4 * quarter;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (n + r >= a.N) continue;
                float v = acc[i][j][r];
                if constexpr (KIND == LIN_GLU) {
                    float u = acc[1][j][r];
                    if (a.bias) { v += a.bias[n + r]; u += a.bias[a.N + n + r]; }
                    v = glu(v, u, a.act);
                } else if constexpr (KIND == LIN_LOW) {
                    if (a.scales) v *= a.scales[adapter];
                } else if (a.bias) v += a.bias[n + r];
                o[n + r] = (O)v;
            }
        }
    }
}

template <typename T, int KIND> drf_status launch(LinArgs& a, bool by_slot, hipStream_t st)
{
    const int columns = KIND == LIN_GLU ? 32 : 64;
    make_fast_div(a.tokens, &a.tok_magic, &a.tok_shift);
    a.slot_rows = by_slot ? a.tokens : a.slots * a.tokens;
    a.tiles_m = (a.slot_rows + 63) / 64;                            // (at most 2^30 rows)
    a.tiles_n = (a.N + columns - 1) / columns;
    a.tiles = (long long)a.tiles_m * a.tiles_n * (by_slot ? a.slots : 1);
    const long long most = 1 << 23;                                 // (a launch holds fewer than 2^32 threads)
    for (a.first = 0; a.first < a.tiles; a.first += most) {
        hipLaunchKernelGGL((linear_kernel<T, KIND>), dim3((unsigned)std::min(most, a.tiles - a.first)), dim3(256), 0, st, a);
        DRF_HIP(hipGetLastError());
    }
    return DRF_OK;
}

constexpr int kMaxColumns = 1 << 20;

drf_status check_columns(const char* what, int n)
{
    if (n < 1) DRF_FAIL(DRF_EINVAL, "%s must be >= 1", what);
    if (n > kMaxColumns) DRF_FAIL(DRF_ESHAPE, "%s must be <= %d", what, kMaxColumns);
    return DRF_OK;
}

drf_status check_io(drf_dtype dtype, int slots, int tokens, int width, int out_width, const drf_rows* x, const drf_rows* out, LinArgs* a)
{
    if (!x || !out || !x->data || !out->data) DRF_FAIL(DRF_EINVAL, "NULL tensor");
    a->x = used_rows(*x, slots, tokens); a->out = used_rows(*out, slots, tokens);
    for (const drf_rows* t : { &a->x, &a->out }) {
        if (t->slot_stride < 0 || t->token_stride < 0) DRF_FAIL(DRF_ESHAPE, "a stride below zero");
        if (t->token_stride >= 1 << 22) DRF_FAIL(DRF_ESHAPE, "a token stride of 2^22 or more");
    }
    if (rows_overlap(a->out, slots, tokens, out_width)) DRF_FAIL(DRF_EINVAL, "rows of the output lie on one another");
    if (a->x.data == a->out.data) DRF_FAIL(DRF_EINVAL, "the output lies on the input");
    if (dtype == DRF_BF16 && (width % 8 || !rows_aligned(a->x, 8))) DRF_FAIL(DRF_ESHAPE, "bf16: width and strides of x must be multiples of 8, x 16-byte aligned");
    a->slots = slots; a->tokens = tokens;
    return DRF_OK;
}

drf_status check_ffn(const drf_gated_ffn_config* cfg)
{
    if (!cfg) DRF_FAIL(DRF_EINVAL, "NULL configuration");
    if (!known_dtype(cfg->dtype)) DRF_FAIL(DRF_EINVAL, "unknown dtype");
    if (cfg->act != DRF_GLU_SILU && cfg->act != DRF_GLU_GELU) DRF_FAIL(DRF_EINVAL, "unknown activation");
    drf_status rc = check_rows_sizes(cfg->slots, cfg->tokens);
    if (rc == DRF_OK) rc = check_columns("width", cfg->width);
    if (rc == DRF_OK) rc = check_columns("hidden", cfg->hidden);
    if (rc == DRF_OK) rc = check_columns("out_width", cfg->out_width);
    if (rc != DRF_OK) return rc;
    if (cfg->dtype == DRF_BF16 && (cfg->width % 8 || cfg->hidden % 8)) DRF_FAIL(DRF_ESHAPE, "bf16: width and hidden must be multiples of 8");
    return DRF_OK;
}

drf_status check_adapters(const drf_adapters_config* cfg)
{
    if (!cfg) DRF_FAIL(DRF_EINVAL, "NULL configuration");
    if (!known_dtype(cfg->dtype)) DRF_FAIL(DRF_EINVAL, "unknown dtype");
    drf_status rc = check_rows_sizes(cfg->slots, cfg->tokens);
    if (rc == DRF_OK) rc = check_columns("width", cfg->width);
    if (rc == DRF_OK) rc = check_columns("out_width", cfg->out_width);
    if (rc != DRF_OK) return rc;
    if (cfg->rank < 1 || cfg->adapters < 0) DRF_FAIL(DRF_EINVAL, "rank must be >= 1 and adapters >= 0");
    if (cfg->rank > 256) DRF_FAIL(DRF_ESHAPE, "rank must be <= 256 (got %d)", cfg->rank);
    if (cfg->dtype == DRF_BF16 && cfg->width % 8) DRF_FAIL(DRF_ESHAPE, "bf16: width must be a multiple of 8");
    return DRF_OK;
}

size_t size_of(drf_dtype t) { return t == DRF_BF16 ? 2 : 4; }
size_t round16(size_t n) { return (n + 15) & ~(size_t)15; }

template <typename T> drf_status run_ffn(const drf_gated_ffn_config& c, LinArgs a, void* scratch, hipStream_t st)
{
    const drf_rows out = a.out, mid = { scratch, (int64_t)c.tokens * c.hidden, c.hidden };
    a.lens = c.lens;
    a.w = c.w_in; a.bias = c.b_in; a.N = c.hidden; a.K = c.width; a.act = c.act; a.out = mid;
    a.in_vec = sizeof(T) == 2 || (c.width % 4 == 0 && rows_aligned(a.x, 4) && aligned16(c.w_in));
    drf_status rc = launch<T, LIN_GLU>(a, false, st);
    if (rc != DRF_OK) return rc;
    a.x = mid; a.out = out;
    a.w = c.w_out; a.bias = c.b_out; a.N = c.out_width; a.K = c.hidden;
    a.in_vec = sizeof(T) == 2 || (c.hidden % 4 == 0 && aligned16(c.w_out));
    return launch<T, LIN_STORE>(a, false, st);
}

template <typename T> drf_status run_adapters(const drf_adapters_config& c, LinArgs a, float* scratch, hipStream_t st)
{
    a.lens = c.lens;
    a.which = c.which; a.adapters = c.adapters; a.rank = c.rank; a.scales = c.scales; a.b = c.b; a.low = scratch;
    a.K = c.width;
    const bool x_vec = sizeof(T) == 2 || (c.width % 4 == 0 && rows_aligned(a.x, 4));
    if (c.adapters) {
        LinArgs l = a;
        l.out = { scratch, (int64_t)c.tokens * c.rank, c.rank };
        l.w = c.a; l.N = c.rank;
        l.in_vec = x_vec && aligned16(c.a);
        const drf_status rc = launch<T, LIN_LOW>(l, true, st);
        if (rc != DRF_OK) return rc;
    }
    a.w = c.w; a.bias = c.bias; a.N = c.out_width;
    a.in_vec = x_vec && aligned16(c.w);
    return launch<T, LIN_ADAPT>(a, false, st);
}

}  // namespace

}  // namespace drf

using namespace drf;

extern "C" size_t drf_gated_ffn_scratch_bytes(const drf_gated_ffn_config* cfg)
{
    if (check_ffn(cfg) != DRF_OK) return 0;
    return round16((size_t)cfg->slots * cfg->tokens * cfg->hidden * size_of(cfg->dtype));
}

extern "C" drf_status drf_gated_ffn(const drf_gated_ffn_config* cfg, const drf_rows* x, const drf_rows* out, void* scratch, size_t scratch_bytes,
                                    void* hip_stream)
{
    drf_status rc = check_ffn(cfg);
    if (rc != DRF_OK) return rc;
    const drf_gated_ffn_config& c = *cfg;
    if (c.slots == 0 || c.tokens == 0) return DRF_OK;
    LinArgs a{};
    if ((rc = check_io(c.dtype, c.slots, c.tokens, c.width, c.out_width, x, out, &a)) != DRF_OK) return rc;
    if (!c.w_in || !c.w_out) DRF_FAIL(DRF_EINVAL, "NULL weights");
    if (c.dtype == DRF_BF16 && (!aligned16(c.w_in) || !aligned16(c.w_out))) DRF_FAIL(DRF_ESHAPE, "bf16 weights must be 16-byte aligned");
    if (!scratch || !aligned16(scratch) || scratch_bytes < drf_gated_ffn_scratch_bytes(cfg)) DRF_FAIL(DRF_EINVAL, "scratch is NULL, not 16-byte aligned or too small");
    return c.dtype == DRF_BF16 ? run_ffn<bf16_t>(c, a, scratch, (hipStream_t)hip_stream) : run_ffn<float>(c, a, scratch, (hipStream_t)hip_stream);
}

extern "C" size_t drf_linear_adapters_scratch_bytes(const drf_adapters_config* cfg)
{
    if (check_adapters(cfg) != DRF_OK || cfg->adapters == 0) return 0;
    return round16((size_t)cfg->slots * cfg->tokens * cfg->rank * sizeof(float));
}

extern "C" drf_status drf_linear_adapters(const drf_adapters_config* cfg, const drf_rows* x, const drf_rows* out, void* scratch, size_t scratch_bytes,
                                          void* hip_stream)
{
    drf_status rc = check_adapters(cfg);
    if (rc != DRF_OK) return rc;
    const drf_adapters_config& c = *cfg;
    if (c.slots == 0 || c.tokens == 0) return DRF_OK;
    LinArgs a{};
    if ((rc = check_io(c.dtype, c.slots, c.tokens, c.width, c.out_width, x, out, &a)) != DRF_OK) return rc;
    if (!c.w) DRF_FAIL(DRF_EINVAL, "NULL weights");
    if (c.adapters && (!c.a || !c.b || !c.which)) DRF_FAIL(DRF_EINVAL, "NULL adapters");
    if (c.dtype == DRF_BF16 && (!aligned16(c.w) || (c.adapters && !aligned16(c.a)))) DRF_FAIL(DRF_ESHAPE, "bf16 weights must be 16-byte aligned");
    if (c.adapters && (!scratch || !aligned16(scratch) || scratch_bytes < drf_linear_adapters_scratch_bytes(cfg)))
        DRF_FAIL(DRF_EINVAL, "scratch is NULL, not 16-byte aligned or too small");
    return c.dtype == DRF_BF16 ? run_adapters<bf16_t>(c, a, (float*)scratch, (hipStream_t)hip_stream)
                               : run_adapters<float>(c, a, (float*)scratch, (hipStream_t)hip_stream);
}
