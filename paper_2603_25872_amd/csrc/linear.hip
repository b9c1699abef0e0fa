// Linears of a block that carry more than a product: the gated feed-forward block and a projection with low-rank adapters of many requests.
//
//   feed-forward   u = x [Wg; Wv]^T + b,  p = act(u_g) u_v  in one launch: a tile of the first product takes the rows of Wg and Wv sixteen and sixteen, so that
//                  a lane ends with gate and value of the same columns;  then out = p Wo^T + b
//   adapters       t = s_i x A_i^T  [row][rank] in one launch;  then out = x W^T + t B_i^T + b: the adapter is `rank` more columns of the product's inner
//                  axis, whose operands are a row's t and its own adapter's B
//
// This file has the entry points, the choice of a tile, x A^T and all of fp32; bf16 products run on the tiles of linear_tile.h.  The weights are the matrix
// instruction's first operand throughout: a lane ends with four consecutive columns of one row.
#include "linear_device.h"
#include "../../include/drf_measure.h"

namespace drf {

namespace {

// ---- x A^T ------------------------------------------------------------------------------------------------
// bf16: 16 MI rows of one slot by 32 of the rank's columns a workgroup, operands straight to registers, the inner axis dealt over NW waves that add up
// through LDS.  Reads x once for every 32 columns of the rank; bound by that.  The sums go out as two bf16 operands: the upper 8 bits of the fp32 value and
// the rest rounded to 8 (2^-16 of the value is lost); one that is no number is itself and zero.
template <int MI, int NW>
__global__ void __launch_bounds__(NW * 64) adapters_low_kernel(const LinArgs a)
{
    constexpr int U = 4;
    __shared__ f32x4 part[NW][2 * MI][64];
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long id = a.first + blockIdx.x;
    const int parts = a.low_cols / 32, slot = (int)(id / ((long long)a.slot_tiles * parts)), in = (int)(id - (long long)slot * a.slot_tiles * parts);
    const int tile = in / parts, r0 = (in - tile * parts) * 32, row0 = tile * 16 * MI;
    const int ad = adapter_of(a, slot), len = slot_len(a.lens, slot, a.tokens);
    if (ad < 0 || row0 >= len) return;
    const bf16_t *x[MI], *w[2];
#pragma unroll
    for (int j = 0; j < MI; ++j) {
        const int token = row0 + 16 * j + l16;
        x[j] = (const bf16_t*)a.x.data + slot * a.x.slot_stride + (token < len ? token : row0) * a.x.token_stride + 8 * quarter;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = r0 + 16 * i + l16;
        w[i] = (const bf16_t*)a.a + ((size_t)ad * a.rank + (r < a.rank ? r : a.rank - 1)) * a.K + 8 * quarter;
    }
    f32x4 acc[2][MI];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < MI; ++j) acc[i][j] = (f32x4){ 0.f, 0.f, 0.f, 0.f };
    const u32x4 zero = { 0, 0, 0, 0 };
    for (int k0 = wave * 32; k0 < a.K; k0 += NW * 32 * U) {
        u32x4 fx[U][MI], fw[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = k0 + u * NW * 32;
            const bool in_row = k + 8 * quarter < a.K;
#pragma unroll
            for (int j = 0; j < MI; ++j) fx[u][j] = in_row ? *reinterpret_cast<const u32x4*>(x[j] + k) : zero;
#pragma unroll
            for (int i = 0; i < 2; ++i) fw[u][i] = in_row ? *reinterpret_cast<const u32x4*>(w[i] + k) : zero;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < MI; ++j) acc[i][j] = mma_bf16(fw[u][i], fx[u][j], acc[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < MI; ++j) part[wave][i * MI + j][lane] = acc[i][j];
    __syncthreads();
    const float scale = a.scales ? a.scales[ad] : 1.f;
    for (int p = wave; p < 2 * MI; p += NW) {
        const int i = p / MI, j = p - i * MI, token = row0 + 16 * j + l16, r = r0 + 16 * i + 4 * quarter;
        f32x4 v = part[0][p][lane];
#pragma unroll
        for (int w2 = 1; w2 < NW; ++w2) v += part[w2][p][lane];
        bf16x4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float t = r + e < a.rank ? v[e] * scale : 0.f;
            const float top = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, t) & 0xffff0000u);
            const bool fine = fabsf(t) < INFINITY;
            hi[e] = (bf16_t)(fine ? top : t);
            lo[e] = (bf16_t)(fine ? t - top : 0.f);
        }
        if (token >= len) continue;
        bf16_t* o = (bf16_t*)a.low + ((size_t)slot * a.tokens + token) * 2 * a.low_cols + r;
        *reinterpret_cast<bf16x4*>(o) = hi;
        *reinterpret_cast<bf16x4*>(o + a.low_cols) = lo;
    }
}

template <int MI, int NW> drf_status launch_low(LinArgs a, hipStream_t st)
{
    a.slot_tiles = (a.tokens + 16 * MI - 1) / (16 * MI);
    a.tiles = (long long)a.slots * a.slot_tiles * (a.low_cols / 32);
    const long long most = 1 << 22;                                 // (a launch holds fewer than 2^32 threads)
    for (a.first = 0; a.first < a.tiles; a.first += most) {
        hipLaunchKernelGGL((adapters_low_kernel<MI, NW>), dim3((unsigned)std::min(most, a.tiles - a.first)), dim3(NW * 64), 0, st, a);
        DRF_HIP(hipGetLastError());
    }
    return DRF_OK;
}

// ---- fp32 -------------------------------------------------------------------------------------------------
// Tiles of 64 rows by 64 rows of the weights on four waves, a wave 32 x 32; 16 elements of the inner axis a step, staged in LDS through registers a step
// ahead.  LIN_LOW: x A^T of one slot.
constexpr int LIN_LOW = 3;

// c += w . x over 16 elements of the inner axis, a lane's four each
__device__ inline void multiply(f32x4& c, const u32x4& w, const u32x4& x)
{
    const f32x4 a = __builtin_bit_cast(f32x4, w), b = __builtin_bit_cast(f32x4, x);
#pragma unroll
    for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[k], b[k], c, 0, 0, 0);
}

template <int KIND>
__global__ void __launch_bounds__(256) linear_f32_kernel(const LinArgs a)
{
    constexpr int E = 4, BK = 16, PITCH = 80;                       // bytes of a row of 64 in LDS: 16 rows on distinct banks
    __shared__ __attribute__((aligned(16))) unsigned char stage[2][128 * PITCH];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave & 1, wn = wave >> 1;
    const long long id = a.first + blockIdx.x;
    const int tm = (int)(id / a.tiles_n), tn = (int)(id - (long long)tm * a.tiles_n);
    const int group = tm / a.slot_tiles, row0 = (tm - group * a.slot_tiles) * 64, n0 = tn * (KIND == LIN_GLU ? 32 : 64);
    // rows that are not there are read as the tile's first and not stored
    int adapter = -1;
    if constexpr (KIND == LIN_LOW) {
        adapter = adapter_of(a, group);
        if (adapter < 0) return;
    }
    if (a.slot_rows == a.tokens && row0 >= slot_len(a.lens, group, a.tokens)) return;

    // staging: thread t copies the 16-byte pieces t % 4 of rows t / 4 of the activations and of the weights
    const int sr = tid >> 2, sc = (tid & 3) * E;
    int s_slot, s_token;
    if (!locate_row(a, group, row0 + sr, s_slot, s_token)) locate_row(a, group, row0, s_slot, s_token);
    const float* xr = (const float*)a.x.data + s_slot * a.x.slot_stride + s_token * a.x.token_stride;
    const float* wr = (const float*)a.w;
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
            for (int j = 0; j < 2; ++j) multiply(acc[i][j], fw[i], fx[j]);
        if (s + 1 < steps) put((s + 1) & 1);
        __syncthreads();
    }

    int slot[2], token[2];
    bool live[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        live[j] = locate_row(a, group, row0 + wm * 32 + j * 16 + l16, slot[j], token[j]);
        if (!live[j]) slot[j] = token[j] = 0;
    }
    if constexpr (KIND == LIN_ADAPT) {
        int first, last, t;
        locate_row(a, group, row0, first, t);
        locate_row(a, group, std::min(row0 + 64, a.slot_rows) - 1, last, t);
        for (int s = first; s <= last; ++s) {                       // (the same for the whole workgroup)
            const int i = adapter_of(a, s);
            if (i < 0) continue;
            const float* b = (const float*)a.b + (size_t)i * a.N * a.rank;
            // into sums of its own, of which the slot's rows take theirs: an infinite weight of one adapter is nothing to the rows of another
            f32x4 sum[2][2];
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int j = 0; j < 2; ++j) sum[p][j] = (f32x4){ 0.f, 0.f, 0.f, 0.f };
            for (int k = 0; k < a.rank; k += BK) {
                u32x4 fw[2], fx[2];
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    int n = n0 + wn * 32 + p * 16 + l16;
                    n = n < a.N ? n : a.N - 1;
                    fw[p] = load16(b + (size_t)n * a.rank, k + quarter * E, a.rank, a.b_vec);
                    fx[p] = (u32x4){ 0, 0, 0, 0 };
                    if (live[p] && slot[p] == s) fx[p] = load16((const float*)a.low + ((size_t)slot[p] * a.tokens + token[p]) * a.low_cols, k + quarter * E, a.rank, a.b_vec);
                }
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int j = 0; j < 2; ++j) multiply(sum[p][j], fw[p], fx[j]);
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
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if (!live[j]) continue;
        float* o = (float*)a.out.data + slot[j] * a.out.slot_stride + token[j] * a.out.token_stride;
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
                o[n + r] = v;
            }
        }
    }
}

template <int KIND> drf_status launch_f32(LinArgs a, bool by_slot, hipStream_t st)
{
    const int columns = KIND == LIN_GLU ? 32 : 64;
    a.slot_rows = by_slot ? a.tokens : a.slots * a.tokens;
    a.slot_tiles = (a.slot_rows + 63) / 64;                         // (at most 2^30 rows)
    a.tiles_n = (a.N + columns - 1) / columns;
    a.tiles = (long long)a.slot_tiles * a.tiles_n * (by_slot ? a.slots : 1);
    const long long most = 1 << 23;                                 // (a launch holds fewer than 2^32 threads)
    for (a.first = 0; a.first < a.tiles; a.first += most) {
        hipLaunchKernelGGL((linear_f32_kernel<KIND>), dim3((unsigned)std::min(most, a.tiles - a.first)), dim3(256), 0, st, a);
        DRF_HIP(hipGetLastError());
    }
    return DRF_OK;
}

// ---- bf16 -------------------------------------------------------------------------------------------------

constexpr int kMaxTokenStride = 1 << 22;           // 256 rows within 2^31 bytes

// Tiles and a time model of a launch of each: base + (per round of workgroups) round + steps * max(lat, c * thr) us, where a round is per_cu workgroups on each of 256
// CUs and c those that share a CU in it.  Least-squares fits to 220 products (16 to 65536 rows, 64 to 9600 columns, an inner axis of 72 to 4800, weights cold);
// the choice by it is within 1 % of the best tile on average, 35 % behind at worst.
struct Tile { int bm, bn, per_cu; double base, round, lat, thr; };
const Tile kLinTiles[] = { { 256, 256, 1, 0.00, 8.15, 1.317, 0 }, { 256, 128, 1, 0.00, 6.01, 0.847, 0 }, { 128, 128, 1, 0.40, 4.08, 0.549, 0 }, { 128, 64, 2, 1.55, 3.36, 0.386, 0.376 },
                           { 64, 128, 2, 1.45, 3.54, 0.385, 0.347 }, { 64, 64, 2, 1.30, 2.97, 0.274, 0.213 }, { 256, 256, 1, 0.00, 11.7, 1.099, 0 }, { 256, 288, 1, 0.00, 13.6, 1.188, 0 } };
constexpr int kTiles = sizeof(kLinTiles) / sizeof(kLinTiles[0]);
thread_local int g_forced_tile = -1;                    // see drf_probe_linear_tile

// Whether tiles of up to 256 rows may cross slots: offsets within one from its first slot on stay below 2^31 bytes.
bool may_cross(const drf_rows& t, int tokens)
{
    const int64_t most = (int64_t)1 << 30;
    return t.slot_stride < most && (tokens - 1) * t.token_stride + (256 / tokens + 2) * t.slot_stride < most;
}

template <int KIND> drf_status launch_bf16(LinArgs a, hipStream_t st)
{
    // rows that lie one behind the other are those of one slot
    if (KIND != LIN_ADAPT && !a.lens && a.slots > 1) {
        const int64_t xt = a.tokens > 1 ? a.x.token_stride : a.x.slot_stride, ot = a.tokens > 1 ? a.out.token_stride : a.out.slot_stride;
        if (a.x.slot_stride == a.tokens * xt && a.out.slot_stride == a.tokens * ot && xt < kMaxTokenStride && ot < kMaxTokenStride) {
            a.x = { a.x.data, 0, xt }; a.out = { a.out.data, 0, ot };
            a.tokens *= a.slots; a.slots = 1;
            make_fast_div(a.tokens, &a.tok_magic, &a.tok_shift);
        }
    }
    a.out_vec = rows_aligned(a.out, 8);
    const bool cross = a.slots > 1 && may_cross(a.x, a.tokens) && may_cross(a.out, a.tokens);
    const int weight_rows = KIND == LIN_GLU ? 2 * a.N : a.N, steps = (a.K + 63) / 64;
    int best = kTiles - 1;
    double best_us = 1e300;
    for (int t = 0; t < kTiles; ++t) {
        const Tile& m = kLinTiles[t];
        const long long tn = (weight_rows + m.bn - 1) / m.bn, by_slot = (long long)a.slots * ((a.tokens + m.bm - 1) / m.bm);
        if (KIND == LIN_GLU && m.bn % 64) continue;                    // (pairs of pieces in a wave)
        const bool large = m.bm * m.bn >= 256 * 256;
        // (the largest tiles have adapters as steps of its loop only, which keeps to a slot)
        const bool keep = !cross || (KIND == LIN_ADAPT && large && a.adapters);
        if (KIND == LIN_ADAPT && large && a.adapters && !a.b_vec) continue;
        const long long tm = keep ? by_slot : std::min(by_slot, ((long long)a.slots * a.tokens + m.bm - 1) / m.bm);
        const long long tiles = tm * tn, full = tiles / (256 * m.per_cu), share = (tiles - full * 256 * m.per_cu + 255) / 256;
        double us = m.base + full * (m.round + steps * std::max(m.lat, m.per_cu * m.thr));
        if (share) us += m.round + steps * std::max(m.lat, share * m.thr);
        if (t == g_forced_tile) { best = t; break; }
        if (us < best_us) { best_us = us; best = t; }
    }
    const Tile& m = kLinTiles[best];
    const int by_slot = a.slots * ((a.tokens + m.bm - 1) / m.bm), crossing = (a.slots * a.tokens + m.bm - 1) / m.bm;
    const bool crosses = cross && crossing < by_slot && !(KIND == LIN_ADAPT && m.bm * m.bn >= 256 * 256 && a.adapters);
    a.in_loop = KIND == LIN_ADAPT && !crosses && a.b_vec;
    a.slot_rows = crosses ? a.slots * a.tokens : a.tokens;
    a.slot_tiles = (a.slot_rows + m.bm - 1) / m.bm;
    a.tiles_m = crosses ? crossing : by_slot;
    a.tiles_n = (weight_rows + m.bn - 1) / m.bn;
    a.tiles = (long long)a.tiles_m * a.tiles_n;
    return launch_linear_tile<KIND>(best, a, st);
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
        if (t->token_stride >= kMaxTokenStride) DRF_FAIL(DRF_ESHAPE, "a token stride of 2^22 or more");
    }
    if (rows_overlap(a->out, slots, tokens, out_width)) DRF_FAIL(DRF_EINVAL, "rows of the output lie on one another");
    if (a->x.data == a->out.data) DRF_FAIL(DRF_EINVAL, "the output lies on the input");
    if (dtype == DRF_BF16 && (width % 8 || !rows_aligned(a->x, 8))) DRF_FAIL(DRF_ESHAPE, "bf16: width and strides of x must be multiples of 8, x 16-byte aligned");
    a->slots = slots; a->tokens = tokens;
    make_fast_div(tokens, &a->tok_magic, &a->tok_shift);
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

int low_columns(const drf_adapters_config& c) { return c.dtype == DRF_BF16 ? (c.rank + 31) / 32 * 32 : c.rank; }

drf_status run_ffn(const drf_gated_ffn_config& c, LinArgs a, void* scratch, hipStream_t st)
{
    const bool bf16 = c.dtype == DRF_BF16;
    const drf_rows out = a.out, mid = { scratch, (int64_t)c.tokens * c.hidden, c.hidden };
    a.w = c.w_in; a.bias = c.b_in; a.N = c.hidden; a.K = c.width; a.act = c.act; a.out = mid;
    a.in_vec = bf16 || (c.width % 4 == 0 && rows_aligned(a.x, 4) && aligned16(c.w_in));
    const drf_status rc = bf16 ? launch_bf16<LIN_GLU>(a, st) : launch_f32<LIN_GLU>(a, false, st);
    if (rc != DRF_OK) return rc;
    a.x = mid; a.out = out;
    a.w = c.w_out; a.bias = c.b_out; a.N = c.out_width; a.K = c.hidden;
    a.in_vec = bf16 || (c.hidden % 4 == 0 && aligned16(c.w_out));
    return bf16 ? launch_bf16<LIN_STORE>(a, st) : launch_f32<LIN_STORE>(a, false, st);
}

drf_status run_adapters(const drf_adapters_config& c, LinArgs a, void* scratch, hipStream_t st)
{
    const bool bf16 = c.dtype == DRF_BF16, x_vec = bf16 || (c.width % 4 == 0 && rows_aligned(a.x, 4));
    a.which = c.which; a.adapters = c.adapters; a.rank = c.rank; a.scales = c.scales; a.a = c.a; a.b = c.b; a.low = scratch;
    a.low_cols = low_columns(c);
    a.b_vec = aligned16(c.b) && c.rank % (bf16 ? 8 : 4) == 0;
    a.K = c.width; a.N = c.out_width;
    if (c.adapters) {
        drf_status rc;
        if (bf16) rc = c.tokens <= 16 ? launch_low<1, 8>(a, st) : launch_low<4, 4>(a, st);
        else {
            LinArgs l = a;
            l.out = { scratch, (int64_t)c.tokens * a.low_cols, a.low_cols };
            l.w = c.a; l.N = c.rank;
            l.in_vec = x_vec && aligned16(c.a);
            rc = launch_f32<LIN_LOW>(l, true, st);
        }
        if (rc != DRF_OK) return rc;
    }
    a.w = c.w; a.bias = c.bias;
    a.in_vec = x_vec && aligned16(c.w);
    return bf16 ? launch_bf16<LIN_ADAPT>(a, st) : launch_f32<LIN_ADAPT>(a, false, st);
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
    a.lens = c.lens;
    return run_ffn(c, a, scratch, (hipStream_t)hip_stream);
}

extern "C" size_t drf_linear_adapters_scratch_bytes(const drf_adapters_config* cfg)
{
    if (check_adapters(cfg) != DRF_OK || cfg->adapters == 0) return 0;
    return round16((size_t)cfg->slots * cfg->tokens * low_columns(*cfg) * sizeof(float));
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
    a.lens = c.lens;
    return run_adapters(c, a, scratch, (hipStream_t)hip_stream);
}

extern "C" int drf_probe_linear_tile(int tile)
{
    g_forced_tile = tile;
    return kTiles;
}
