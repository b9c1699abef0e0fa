// Linears of a block that carry more than a product: the gated feed-forward block and a projection with low-rank adapters of many requests.
//
//   feed-forward   u = x [Wg; Wv]^T + b,  p = act(u_g) u_v  in one launch: a tile of the first product takes the rows of Wg and Wv sixteen and sixteen, so that
//                  a lane ends with gate and value of the same columns;  then out = p Wo^T + b
//   adapters       t = s_i x A_i^T  [row][rank] in one launch;  then out = x W^T + t B_i^T + b: the adapter is `rank` more columns of the product's inner
//                  axis, whose operands are a row's t and its own adapter's B
//
// This file has the entry points, the choice of a tile or form, x A^T and the tile of fp32; bf16 products run on the tiles of linear_tile.h and linear_wide.h, few rows
// of both types on the forms of linear_direct.h.  The weights are the matrix
// instruction's first operand throughout: a lane ends with four consecutive columns of one row.
#include "linear_direct.h"
#include "../../include/drf_measure.h"

namespace drf {

namespace {

constexpr int kMaxTokenStride = 1 << 22;           // 256 rows within 2^31 bytes

// Tiles and a time model of a launch of each: base + (per round of workgroups) round + steps * max(lat, c * thr) us, where a round is per_cu workgroups on each of 256
// CUs and c those that share a CU in it.  Least-squares fits to 260 products (16 to 65536 rows, 64 to 9600 columns, an inner axis of 72 to 4800, weights cold).
// The whole choice, tiles and forms, on 300 other products that are drawn (60 of each type, with and without adapters): 1.4 to 3.1 % behind the best on average, a tenth of
// them by more than 7 to 15 %, at worst 28 % (bf16), 35 % (bf16, ranks that are no multiple of 8) and 37 % (fp32), all of these products of 6 to 15 us.
struct Tile { int bm, bn, per_cu; double base, round, lat, thr; };
const Tile kLinTiles[] = { { 256, 256, 1, 0.00, 9.05, 1.075, 0 }, { 256, 128, 1, 0.00, 6.40, 0.723, 0 }, { 128, 128, 1, 0.43, 4.47, 0.451, 0 }, { 128, 64, 2, 1.54, 3.59, 0.324, 0.324 },
                           { 64, 128, 2, 1.60, 3.50, 0.333, 0.333 }, { 64, 64, 2, 1.75, 2.83, 0.207, 0.207 }, { 256, 256, 1, 0.00, 11.9, 0.965, 0 }, { 256, 288, 1, 0.00, 13.6, 1.067, 0 } };
constexpr int kTiles = sizeof(kLinTiles) / sizeof(kLinTiles[0]);
// The forms for few rows of linear_direct.h, rows and weight rows a workgroup in sixteens and its waves: fixed + turns * turn + max(0, workgroups / 256 - hidden) * (group + 128-byte
// pieces of the inner axis * piece) us, fitted likewise (140 and 100 products of 1 to 4096 rows).  The last form's are set by hand: it is looked at up to one workgroup a CU alone,
// where it has no shares to tell apart, and its adapters' share is the first form's.
struct Form { int mi, ni, nw; double fixed, turn, hidden, group, piece; };
constexpr int kForms = 6;
const Form kFormsBf16[kForms] = { { 1, 1, 16, 1.83, 1.13, 0.27, 1.18, 0.095 }, { 1, 4, 8, 1.84, 1.75, 0.40, 0.80, 0.282 }, { 2, 2, 8, 2.18, 1.03, 0.06, 0.85, 0.196 }, { 4, 2, 8, 2.47, 1.47, 0.37, 1.71, 0.343 },
                                  { 1, 2, 8, 2.08, 0.93, 0.25, 0.66, 0.161 }, { 1, 1, 16, 2.0, 1.3, 0, 0, 0 } /* 8 rows by 8, see below */ };
const Form kFormsF32[kForms] = { { 1, 1, 16, 1.80, 1.40, 0.28, 1.40, 0.104 }, { 0 } /* (never ahead) */, { 2, 2, 8, 2.21, 1.84, 0.34, 1.57, 0.254 }, { 4, 2, 8, 2.31, 3.18, 0.34, 2.68, 0.459 },
                                 { 1, 2, 8, 2.10, 1.02, 0.0, 0.71, 0.164 }, { 0 } };
const Tile kTileF32 = { 64, 64, 4, 0.0, 3.67, 0.692, 0.630 };      // steps of 32

double tile_us(const Tile& m, long long tiles, int steps)
{
    const long long full = tiles / (256 * m.per_cu), share = (tiles - full * 256 * m.per_cu + 255) / 256;
    return m.base + full * (m.round + steps * std::max(m.lat, m.per_cu * m.thr)) + (share ? m.round + steps * std::max(m.lat, share * m.thr) : 0.0);
}

// What adapters add, x A^T's launch included: first + pieces of 8 of the rank * rank + workgroups / 256 * (group + pieces * group_rank) us for a form (fitted to products of
// 1 to 800 rows of 1 to 40 slots, ranks of 8 to 128, 4 % off on average; unaligned rows of B count 1.7 times).  It matters most where every row is a slot (200 x 384 x 1152,
// rank 128, fp32, four adapters among the slots: 34 us, on the tile 245; an adapter each: 65 and 352).
struct FormAdapters { double first, rank, group, group_rank; };
const FormAdapters kAdaptBf16[kForms] = { { 1.96, 0.232, 0, 0.246 }, { 2.36, 0.422, 0.476, 0.07 }, { 2.32, 0.401, 0.492, 0.075 }, { 2.39, 0.80, 0.69, 0.1 }, { 2.13, 0.306, 0.165, 0.219 }, { 1.96, 0.232, 0, 0.246 } };
const FormAdapters kAdaptF32[kForms] = { { 2.65, 0.307, 0.066, 0.35 }, { 0 }, { 2.81, 0.491, 0.563, 0.072 }, { 2.78, 0.848, 0.3, 0.05 }, { 2.59, 0.359, 0.153, 0.25 }, { 0 } };

// The same for the bf16 tiles: steps of the loop, or behind it a lane's elements one by one (slots shorter than 16 rows), or slot after slot.
double tile_adapters_us(const Tile& m, const LinArgs& a, long long tiles, bool crosses)
{
    const double rounds = (double)((tiles + 256 * m.per_cu - 1) / (256 * m.per_cu));
    const int pieces = m.bm * m.bn >= 128 * 64 ? 8 : 4, eights = (a.rank + 7) / 8, steps = (a.rank + 31) / 32;     // of 16 x 16 in a wave's tile
    if (!crosses && a.b_vec) return 2.5 + 0.2 * steps;
    if (a.tokens < 16) return rounds * (4.5 + 0.4 * pieces * eights * (a.b_vec ? 1.0 : 3.5));
    return rounds * (4 + 0.25 * pieces + 0.11 * pieces * steps * (crosses ? std::min(a.slots, 31 / a.tokens + 2) : 1) + (a.b_vec ? 0 : 3));
}

// The form with the least modelled time, and that time.
template <typename T, int KIND> int pick_form(const LinArgs& a, double* us)
{
    const Form* forms = sizeof(T) == 2 ? kFormsBf16 : kFormsF32;
    const long long rows = (long long)a.slots * a.tokens, weight_rows = KIND == LIN_GLU ? 2LL * a.N : a.N;
    const int pieces = (a.K * (int)sizeof(T) + 127) / 128;
    int best = 0;
    *us = 1e300;
    for (int f = 0; f < kForms; ++f) {
        const Form& m = forms[f];
        if (!m.mi) continue;
        // the last form takes 8 rows by 8 and twice the pieces a turn.  Up to one workgroup a CU it is what few columns of a long inner axis want (weights cold, 16 by 16 and 8 by 8:
        // 1 x 4608 x 1152 7.9 and 6.2 us, 1 x 9216 x 1152 13.5 and 9.4, 8 x 4608 x 1152 9.4 and 7.7), behind it every other is ahead (1 x 4608 x 2304 7.7 and 10.8)
        const int split = f == kForms - 1 ? 2 : 1, mr = 16 / split * m.mi, nr = 16 / split * m.ni, at_once = m.nw * split;
        const double groups = (double)((rows + mr - 1) / mr) * ((weight_rows + nr - 1) / nr);
        if (split > 1 && (KIND == LIN_GLU || groups > 256)) continue;
        double t = m.fixed + (pieces + at_once - 1) / at_once * m.turn + std::max(0.0, groups / 256 - m.hidden) * (m.group + pieces * m.piece);
        if (KIND == LIN_ADAPT && a.adapters) {
            const FormAdapters& p = (sizeof(T) == 2 ? kAdaptBf16 : kAdaptF32)[f];
            const double eights = (a.rank + 7) / 8 * (sizeof(T) == 2 && !a.b_vec ? 1.7 : 1.0);
            t += p.first + eights * p.rank + groups / 256 * (p.group + eights * p.group_rank);
        }
        if (t < *us) { *us = t; best = f; }
    }
    return best;
}
thread_local int g_forced_tile = -1;                    // see drf_probe_linear_tile
thread_local int g_route[3] = { -1, -1, -1 };           // see drf_probe_linear_route

// ---- x A^T ------------------------------------------------------------------------------------------------
// 16 MI rows of one slot by 32 of the rank's columns a workgroup, operands straight to registers, the inner axis dealt over NW waves, 128 bytes of it at a
// time with U turns on the way (U = 0: all at once), that add up through LDS.  Reads x once for every 32 columns of the rank; bound by that: 65536 x 1152 47 us, 3.2 TB/s (on two and one
// pieces of rows a workgroup 51 and 65), 64 rows of as many requests 5.  fp32 sums go out as they are, for bf16
// as two operands: the upper 8 bits of the next fp32 value towards zero, and the rest rounded to 8 (2^-16 of the value is lost).  So neither is zero and both have the
// value's sign: times an infinite weight they are that infinity.  A zero, an infinity and what is no number are themselves twice.
template <typename T, int MI, int NW, int U>
__global__ void __launch_bounds__(NW * 64) adapters_low_kernel(const LinArgs a)
{
    constexpr int E = 16 / sizeof(T);
    __shared__ f32x4 part[NW][2 * MI][64];
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long id = a.first + blockIdx.x;
    const int parts = (a.rank + 31) / 32, slot = (int)(id / ((long long)a.slot_tiles * parts)), in = (int)(id - (long long)slot * a.slot_tiles * parts);
    const int tile = in / parts, r0 = (in - tile * parts) * 32, row0 = tile * 16 * MI;
    const int ad = adapter_of(a, slot), len = slot_len(a.lens, slot, a.tokens);
    if (ad < 0 || row0 >= len) return;
    const T *x[MI], *w[2];
#pragma unroll
    for (int j = 0; j < MI; ++j) {
        const int token = row0 + 16 * j + l16;
        x[j] = (const T*)a.x.data + slot * a.x.slot_stride + (token < len ? token : row0) * a.x.token_stride;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = r0 + 16 * i + l16;
        w[i] = (const T*)a.a + ((size_t)ad * a.rank + (r < a.rank ? r : a.rank - 1)) * a.K;
    }
    f32x4 acc[2][MI];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < MI; ++j) acc[i][j] = (f32x4){ 0.f, 0.f, 0.f, 0.f };
    if constexpr (U > 0) direct_product<T, MI, 2, NW, U>(acc, x, w, a.K, wave, quarter);
    else if (wave == 0)                             // (rows of less than 16 bytes)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < MI; ++j) acc[i][j] = mma(load_row16(w[i], quarter * E, a.K), load_row16(x[j], quarter * E, a.K), acc[i][j], T{});
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
        if (token >= len) continue;
        const size_t row = (size_t)slot * a.tokens + token;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (r + e < a.rank) ((float*)a.low)[row * a.low_cols + r + e] = v[e] * scale;
        } else {
            bf16x4 hi, lo;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float t = r + e < a.rank ? v[e] * scale : 0.f;
                const float top = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, t) - 1u) & 0xffff0000u);
                const bool fine = fabsf(t) > 0.f && fabsf(t) < INFINITY;
                hi[e] = (bf16_t)(fine ? top : t);
                lo[e] = (bf16_t)(fine ? t - top : t);
            }
            bf16_t* o = (bf16_t*)a.low + row * 2 * a.low_cols + r;
            *reinterpret_cast<bf16x4*>(o) = hi;
            *reinterpret_cast<bf16x4*>(o + a.low_cols) = lo;
        }
    }
}

template <typename T, int MI, int NW, int U> drf_status launch_low(LinArgs a, hipStream_t st)
{
    a.slot_tiles = (a.tokens + 16 * MI - 1) / (16 * MI);
    a.tiles = (long long)a.slots * a.slot_tiles * ((a.rank + 31) / 32);
    const long long most = 1 << 22;                                 // (a launch holds fewer than 2^32 threads)
    for (a.first = 0; a.first < a.tiles; a.first += most) {
        hipLaunchKernelGGL((adapters_low_kernel<T, MI, NW, U>), dim3((unsigned)std::min(most, a.tiles - a.first)), dim3(NW * 64), 0, st, a);
        DRF_HIP(hipGetLastError());
    }
    return DRF_OK;
}

template <typename T> drf_status run_low(const LinArgs& a, hipStream_t st)
{
    if constexpr (sizeof(T) == 4) {
        if (a.K < 4) return launch_low<T, 1, 1, 0>(a, st);
    }
    return a.tokens <= 16 ? launch_low<T, 1, 8, 3>(a, st) : (long long)a.slots * ((a.tokens + 63) / 64) < 512 ? launch_low<T, 2, 8, 3>(a, st) : launch_low<T, 4, 4, 3>(a, st);
}

// ---- fp32 -------------------------------------------------------------------------------------------------
// Tiles of 64 rows by 64 rows of the weights on four waves, a wave 32 x 32; 32 elements of the inner axis a step, staged in LDS through registers DEPTH steps ahead, 16
// bytes at a time at any address.  Bound by the matrix unit where it has enough tiles: 2241 x 3502 x 2153 319 us (106 of 157 TFLOP/s; 128 x 128 tiles 297, but slower below).
template <int KIND>
__global__ void __launch_bounds__(256) linear_f32_kernel(const LinArgs a)
{
    constexpr int W = 2, DEPTH = 2, BM = 32 * W, PITCH = 144, Q = BM / 32;       // pieces of a wave's side; bytes of a row of 128 in LDS; pieces of a thread
    __shared__ __attribute__((aligned(16))) unsigned char stage[2 * 2 * BM * PITCH];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave & 1, wn = wave >> 1;
    const long long id = a.first + blockIdx.x;
    const int tm = (int)(id / a.tiles_n), tn = (int)(id - (long long)tm * a.tiles_n);
    const int row0 = tm * BM, n0 = tn * (KIND == LIN_GLU ? BM / 2 : BM);
    if (a.slots == 1 && row0 >= slot_len(a.lens, 0, a.tokens)) return;

    // staging: thread t copies piece t % 8 of rows t / 8 + 32 i of the activations and of the weights; rows that are not there are read as slot 0's first and not stored
    const float *xr[Q], *wr[Q];
    const int sc = (tid & 7) * 4;
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        const int r = tid / 8 + 32 * i;
        int slot, token;
        locate_row(a, 0, row0 + r, slot, token);
        if (row0 + r >= a.slot_rows) slot = token = 0;
        xr[i] = (const float*)a.x.data + slot * a.x.slot_stride + token * a.x.token_stride + sc;
        int n = n0 + (KIND == LIN_GLU ? r / 32 * 16 + r % 16 : r);
        n = n < a.N ? n : a.N - 1;
        wr[i] = (const float*)a.w + ((size_t)n + (KIND == LIN_GLU && r / 16 % 2 ? a.N : 0)) * a.K + sc;
    }
    typedef float piece __attribute__((ext_vector_type(4), aligned(4)));
    u32x4 px[DEPTH][Q], pw[DEPTH][Q];
    auto fetch = [&](int d, int s) __attribute__((always_inline)) {
        if (s * 32 + 32 <= a.K) {
#pragma unroll
            for (int i = 0; i < Q; ++i) {
                px[d][i] = __builtin_bit_cast(u32x4, *reinterpret_cast<const piece*>(xr[i] + s * 32));
                pw[d][i] = __builtin_bit_cast(u32x4, *reinterpret_cast<const piece*>(wr[i] + s * 32));
            }
        } else
#pragma unroll
            for (int i = 0; i < Q; ++i) {
                px[d][i] = load_row16(xr[i] - sc, s * 32 + sc, a.K);
                pw[d][i] = load_row16(wr[i] - sc, s * 32 + sc, a.K);
            }
    };
    auto put = [&](int d, int s) __attribute__((always_inline)) {
        unsigned char* st = stage + (s & 1) * 2 * BM * PITCH + (tid & 7) * 16;
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            *reinterpret_cast<u32x4*>(st + (tid / 8 + 32 * i) * PITCH) = px[d][i];
            *reinterpret_cast<u32x4*>(st + (BM + tid / 8 + 32 * i) * PITCH) = pw[d][i];
        }
    };
    f32x4 acc[W][W];                                                // [weight piece][activation piece]
#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
        for (int j = 0; j < W; ++j) acc[i][j] = (f32x4){ 0.f, 0.f, 0.f, 0.f };
    const int steps = (a.K + 31) / 32;
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (d < steps) fetch(d, d);
    for (int s0 = 0; s0 < steps; s0 += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int s = s0 + d;
            if (s >= steps) break;
            put(d, s);
            __syncthreads();                                        // (the other stage is written again only behind the next one)
            if (s + DEPTH < steps) fetch(d, s + DEPTH);
            const unsigned char* st = stage + (s & 1) * 2 * BM * PITCH;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 fx[W], fw[W];
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    fx[i] = *reinterpret_cast<const u32x4*>(st + (wm * 16 * W + i * 16 + l16) * PITCH + (4 * h + quarter) * 16);
                    fw[i] = *reinterpret_cast<const u32x4*>(st + (BM + wn * 16 * W + i * 16 + l16) * PITCH + (4 * h + quarter) * 16);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int i = 0; i < W; ++i)
#pragma unroll
                        for (int j = 0; j < W; ++j)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f32x4, fw[i])[k], __builtin_bit_cast(f32x4, fx[j])[k], acc[i][j], 0, 0, 0);
            }
        }
    }

    int slot[W], token[W];
    bool live[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
        live[j] = locate_row(a, 0, row0 + (wm * W + j) * 16 + l16, slot[j], token[j]);
        if (!live[j]) slot[j] = token[j] = 0;
    }
    if (KIND == LIN_ADAPT && a.adapters) {
        int first, last, t;
        locate_row(a, 0, row0 + wm * 16 * W, first, t);
        locate_row(a, 0, std::min(row0 + (wm + 1) * 16 * W, a.slot_rows) - 1, last, t);
        for (int s = first; s <= last; ++s) {                       // (the same for the whole wave)
            const int ad = adapter_of(a, s);
            if (ad < 0) continue;
            const float* b = (const float*)a.b + (size_t)ad * a.N * a.rank;
            // into sums of its own, of which the slot's rows take theirs: an infinite weight of one adapter is nothing to the rows of another
#pragma unroll
            for (int j = 0; j < W; ++j) {
                f32x4 sum[W];
#pragma unroll
                for (int i = 0; i < W; ++i) sum[i] = (f32x4){ 0.f, 0.f, 0.f, 0.f };
                for (int k = 0; k < a.rank; k += 16) {
                    u32x4 fx = { 0, 0, 0, 0 };
                    if (live[j] && slot[j] == s) fx = load_row16((const float*)a.low + ((size_t)slot[j] * a.tokens + token[j]) * a.low_cols, k + quarter * 4, a.rank);
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        int n = n0 + (wn * W + i) * 16 + l16;
                        n = n < a.N ? n : a.N - 1;
                        sum[i] = mma(load_row16(b + (size_t)n * a.rank, k + quarter * 4, a.rank), fx, sum[i], 0.f);
                    }
                }
#pragma unroll
                for (int i = 0; i < W; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j][r] += slot[j] == s ? sum[i][r] : 0.f;
            }
        }
    }

    // acc[i][j][r] is (row 16 j + l16, weight row 16 i + 4 quarter + r) of the wave's tile
#pragma unroll
    for (int j = 0; j < W; ++j) {
        if (!live[j]) continue;
        float* o = (float*)a.out.data + slot[j] * a.out.slot_stride + token[j] * a.out.token_stride;
#pragma unroll
        for (int i = 0; i < W; i += KIND == LIN_GLU ? 2 : 1) {
            const int n = n0 + (KIND == LIN_GLU ? (wn * W + i) * 8 : (wn * W + i) * 16) + 4 * quarter;
            f32x4 v = acc[i][j];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int c = n + r < a.N ? n + r : a.N - 1;
                if constexpr (KIND == LIN_GLU) {
                    float u = acc[i + 1][j][r];
                    if (a.bias) { v[r] += a.bias[c]; u += a.bias[a.N + c]; }
                    v[r] = glu(v[r], u, a.act);
                } else if (a.bias) v[r] += a.bias[c];
            }
            if (n + 4 <= a.N) *reinterpret_cast<piece*>(o + n) = v;
            else
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (n + r < a.N) o[n + r] = v[r];
        }
    }
}

template <int KIND> drf_status launch_f32_tiles(LinArgs a, hipStream_t st)
{
    constexpr int BM = 64, columns = KIND == LIN_GLU ? BM / 2 : BM;
    a.slot_rows = a.slots * a.tokens;
    a.tiles_n = (a.N + columns - 1) / columns;
    a.tiles = (long long)((a.slot_rows + BM - 1) / BM) * a.tiles_n;     // (at most 2^30 rows)
    const long long most = 1 << 23;                                 // (a launch holds fewer than 2^32 threads)
    for (a.first = 0; a.first < a.tiles; a.first += most) {
        hipLaunchKernelGGL((linear_f32_kernel<KIND>), dim3((unsigned)std::min(most, a.tiles - a.first)), dim3(256), 0, st, a);
        DRF_HIP(hipGetLastError());
    }
    return DRF_OK;
}

template <int KIND> drf_status launch_f32(const LinArgs& a, hipStream_t st)
{
    double us;
    const int form = pick_form<float, KIND>(a, &us), forced = g_forced_tile - kTiles;
    auto direct = [&](int f) { g_route[KIND] = kTiles + f; return launch_linear_direct<float, KIND>(f, a, st); };
    if (forced >= 0 && forced < kForms && kFormsF32[forced].mi && a.K >= 4) return direct(forced);     // (rows of at least 16 bytes)
    const long long tiles = ((long long)a.slots * a.tokens + 63) / 64 * (((KIND == LIN_GLU ? 2LL * a.N : a.N) + 63) / 64);
    double tile = tile_us(kTileF32, tiles, (a.K + 31) / 32);
    if (KIND == LIN_ADAPT && a.adapters) {                          // slot after slot of a wave's 32 rows
        const int reach = std::min(std::min(a.slots, 32), 31 / a.tokens + 1 + (a.tokens > 1));
        tile += 1.1 + 1.1 * std::max(1.0, tiles / 256.0) + reach * (0.42 + 0.64 * ((a.rank + 15) / 16)) * (double)((tiles + 1023) / 1024);
    }
    if (forced != kForms && a.K >= 4 && us < tile) return direct(form);
    g_route[KIND] = kTiles + kForms;
    return launch_f32_tiles<KIND>(a, st);
}

// ---- bf16 -------------------------------------------------------------------------------------------------

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
        const bool large = m.bm * m.bn >= 256 * 128;
        // (the largest tiles have adapters as steps of their loop only, and then keep to a slot)
        const bool keep = !cross || (KIND == LIN_ADAPT && large && a.adapters);
        if (KIND == LIN_ADAPT && large && a.adapters && !a.b_vec) continue;
        const long long tm = keep ? by_slot : std::min(by_slot, ((long long)a.slots * a.tokens + m.bm - 1) / m.bm);
        const bool crosses = !keep && tm < by_slot;
        double us = tile_us(m, tm * tn, steps + (KIND == LIN_ADAPT && a.adapters && !crosses && a.b_vec ? a.low_cols / 32 : 0));
        if (KIND == LIN_ADAPT && a.adapters) us += tile_adapters_us(m, a, tm * tn, crosses);
        if (t == g_forced_tile) { best = t; break; }
        if (us < best_us) { best_us = us; best = t; }
    }
    double form_us;
    const int form = pick_form<bf16_t, KIND>(a, &form_us), forced = g_forced_tile - kTiles;
    auto direct = [&](int f) { g_route[KIND] = kTiles + f; return launch_linear_direct<bf16_t, KIND>(f, a, st); };
    if (forced >= 0 && forced < (KIND == LIN_GLU ? kForms - 1 : kForms)) return direct(forced);
    if (g_forced_tile < 0 && form_us < best_us) return direct(form);
    g_route[KIND] = best;
    const Tile& m = kLinTiles[best];
    const int by_slot = a.slots * ((a.tokens + m.bm - 1) / m.bm), crossing = (a.slots * a.tokens + m.bm - 1) / m.bm;
    const bool crosses = cross && crossing < by_slot && !(KIND == LIN_ADAPT && m.bm * m.bn >= 256 * 128 && a.adapters);
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
    const drf_status rc = bf16 ? launch_bf16<LIN_GLU>(a, st) : launch_f32<LIN_GLU>(a, st);
    if (rc != DRF_OK) return rc;
    a.x = mid; a.out = out;
    a.w = c.w_out; a.bias = c.b_out; a.N = c.out_width; a.K = c.hidden;
    return bf16 ? launch_bf16<LIN_STORE>(a, st) : launch_f32<LIN_STORE>(a, st);
}

drf_status run_adapters(const drf_adapters_config& c, LinArgs a, void* scratch, hipStream_t st)
{
    const bool bf16 = c.dtype == DRF_BF16;
    a.which = c.which; a.adapters = c.adapters; a.rank = c.rank; a.scales = c.scales; a.a = c.a; a.b = c.b; a.low = scratch;
    a.low_cols = low_columns(c);
    a.b_vec = aligned16(c.b) && c.rank % 8 == 0;
    a.K = c.width; a.N = c.out_width;
    if (c.adapters) {
        const drf_status rc = bf16 ? run_low<bf16_t>(a, st) : run_low<float>(a, st);
        if (rc != DRF_OK) return rc;
    }
    a.w = c.w; a.bias = c.bias;
    return bf16 ? launch_bf16<LIN_ADAPT>(a, st) : launch_f32<LIN_ADAPT>(a, st);
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
    return kTiles + kForms + 1;
}

extern "C" int drf_probe_linear_route(int product) { return product >= 0 && product < 3 ? g_route[product] : -1; }
