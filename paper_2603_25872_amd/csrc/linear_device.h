// Device code and arguments shared by the kernels of the Linears around a block (linear.hip, linear_tile.h).
#pragma once
#include <algorithm>
#include <type_traits>

#include "gemm_device.h"
#include "rows.h"

namespace drf {

enum { LIN_STORE = 0, LIN_GLU = 1, LIN_ADAPT = 2 };

struct LinArgs {
    drf_rows x, out;
    const void* w;                      // [N][K]; LIN_GLU: [2 N][K], gates and then values
    const float* bias;                  // [N] (LIN_GLU: [2 N]) or NULL
    const int32_t* lens;
    int slots, tokens, N, K;
    uint32_t tok_magic; int tok_shift;
    int slot_rows;                      // rows that are counted together: tokens (tiles do not cross slots) or slots * tokens
    int tiles_m, tiles_n;               // tiles of all rows; tiles of columns
    int slot_tiles;                     // tiles of rows that are counted together
    long long first, tiles;             // tile that this launch begins with; all of them
    int act, out_vec;
    // adapters
    const int32_t* which;
    const float* scales;
    const void* a;                      // [adapters][rank][K]
    const void* b;                      // [adapters][N][rank]
    void* low;                          // x A^T of every row, scaled: fp32 [rank]; for bf16 operands [2][low_cols], upper and lower 8 bits, zeros from rank on
    int adapters, rank, low_cols, b_vec;
    int in_loop;                        // bf16: tiles keep to a slot and B's rows are 16-byte pieces, the adapter is steps of the product's loop
};

namespace {

__device__ inline float glu(float a, float v, int act)
{
    if (act == DRF_GLU_GELU) return gelu_tanh(a) * v;
    return a * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * a)) * v;
}

__device__ inline int adapter_of(const LinArgs& a, int slot)
{
    const int i = a.adapters ? a.which[slot] : -1;
    return i >= 0 && i < a.adapters ? i : -1;
}

// Row m of the rows that are counted together, of group `group` of them: its slot and token; false where it is not there or behind its slot's length.
__device__ inline bool locate_row(const LinArgs& a, int group, int m, int& slot, int& token)
{
    if (a.slot_rows == a.tokens) { slot = group; token = m; }
    else { slot = fast_div(m, a.tok_magic, a.tok_shift); token = m - slot * a.tokens; }
    return m < a.slot_rows && token < slot_len(a.lens, slot, a.tokens);
}

typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
__device__ inline f32x4 mma_bf16(const u32x4& w, const u32x4& x, const f32x4& c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
}

// 16 bytes of a row of n elements from element k on, zeros behind its end
template <typename T> __device__ inline u32x4 load16(const T* row, int k, int n, bool vec)
{
    constexpr int E = 16 / sizeof(T);
    if (vec) return k < n ? *reinterpret_cast<const u32x4*>(row + k) : (u32x4){ 0, 0, 0, 0 };
    T v[E];
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = k + j < n ? row[k + j] : (T)0.f;
    u32x4 r;
    __builtin_memcpy(&r, v, 16);
    return r;
}

// The bias of a tile's BN weight rows into LDS, by copies of 4 bytes a lane where there is one (nothing waits for them before the first step's copies, which are
// younger) and zeros where there is none.  Whole 64s of them are written.
template <int BN, int NW, int KIND> __device__ __forceinline__ void stage_bias(const LinArgs& a, float* bias, int n0, int wave)
{
    const int lane = threadIdx.x & 63;
    if (!a.bias) {
        for (int t = threadIdx.x; t < BN; t += NW * 64) bias[t] = 0.f;
        return;
    }
#pragma unroll
    for (int c = 0; c < (BN + 64 * NW - 1) / (64 * NW); ++c) {
        const int piece = c * NW + wave, t = piece * 64 + lane;
        if (piece * 64 >= BN) continue;
        int n = KIND == LIN_GLU ? t / 32 * 16 + t % 16 : t;
        n = n0 + n < a.N ? n0 + n : a.N - 1;
        if constexpr (KIND == LIN_GLU) n += t / 16 % 2 ? a.N : 0;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
                     :: "s"((uint32_t)(uintptr_t)(DRF_LDS_AS float*)bias + (uint32_t)piece * 256u), "v"((uint32_t)n * 4u), "s"(a.bias) : "memory");
    }
}

// What the adapters add to a wave's tile: acc[i][j][r] is (row mw + 16 j + l16, column nw + 16 i + 4 quarter + r) of the group's rows.
// A slot's product goes into sums of its own, of which its rows take theirs: an infinite weight of one adapter is nothing to the rows of another.  Where slots
// are shorter than a tile's sixteen rows a lane adds up its elements one by one, each row from its own adapter, read once.
template <int MI, int NI>
__device__ __forceinline__ void add_adapters(f32x4 (&acc)[NI][MI], const LinArgs& a, int group, int mw, int nw)
{
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4, LC = a.low_cols;
    if (!a.adapters) return;
    if (a.tokens < 16) {
        bool some[MI];
        const bf16_t *t[MI], *b0[MI];
#pragma unroll
        for (int j = 0; j < MI; ++j) {                              // (all rows' adapters, then all their loads beside one another; those of a row without one are some row's)
            int slot, token;
            some[j] = locate_row(a, group, mw + 16 * j + l16, slot, token);
            if (!some[j]) slot = token = 0;
            const int ad = adapter_of(a, slot);
            some[j] = some[j] && ad >= 0;
            t[j] = (const bf16_t*)a.low + ((size_t)slot * a.tokens + token) * 2 * LC;
            b0[j] = (const bf16_t*)a.b + (size_t)(ad < 0 ? 0 : ad) * a.N * a.rank;
        }
        constexpr int JG = NI <= 2 ? 2 : 1;                         // rows' pieces at a time
#pragma unroll
        for (int j0 = 0; j0 < MI; j0 += JG)
            for (int k = 0; k < a.rank; k += 8) {
                bf16x8 hi[JG], lo[JG];
                u32x4 f[JG][NI][4];
#pragma unroll
                for (int j = 0; j < JG; ++j) {
                    hi[j] = *reinterpret_cast<const bf16x8*>(t[j0 + j] + k);
                    lo[j] = *reinterpret_cast<const bf16x8*>(t[j0 + j] + LC + k);
#pragma unroll
                    for (int i = 0; i < NI; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int n = nw + 16 * i + 4 * quarter + r;
                            f[j][i][r] = load16(b0[j0 + j] + (size_t)(n < a.N ? n : a.N - 1) * a.rank, k, a.rank, a.b_vec);
                        }
                }
#pragma unroll
                for (int j = 0; j < JG; ++j) {
                    float low[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) low[e] = (float)hi[j][e] + (float)lo[j][e];
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            float v = 0.f;
#pragma unroll
                            for (int e = 0; e < 8; ++e) v = fmaf(low[e], (float)__builtin_bit_cast(bf16x8, f[j][i][r])[e], v);
                            acc[i][j0 + j][r] += some[j0 + j] ? v : 0.f;
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        return;
    }
    auto slot_of = [&](int m) { return a.slot_rows == a.tokens ? group : fast_div(m < a.slot_rows ? m : a.slot_rows - 1, a.tok_magic, a.tok_shift); };
    auto low_row = [&](int m) {                                     // (a row that is not there: some row's, its result is not stored)
        int slot, token;
        if (!locate_row(a, group, m, slot, token)) { slot = slot_of(m); token = 0; }
        return (const bf16_t*)a.low + ((size_t)slot * a.tokens + token) * 2 * LC;
    };
    auto b_frag = [&](int ad, int i, int k) {
        int n = nw + 16 * i + l16;
        n = n < a.N ? n : a.N - 1;
        return load16((const bf16_t*)a.b + ((size_t)ad * a.N + n) * a.rank, k + 8 * quarter, a.rank, a.b_vec);
    };
    if (slot_of(mw) == slot_of(mw + 16 * MI - 1)) {                 // one slot: straight into the tile's sums
        const int ad = adapter_of(a, slot_of(mw));
        if (ad < 0) return;
        const bf16_t* t[MI];
#pragma unroll
        for (int j = 0; j < MI; ++j) t[j] = low_row(mw + 16 * j + l16) + 8 * quarter;
        for (int k = 0; k < LC; k += 32) {
            u32x4 hi[MI], lo[MI];
#pragma unroll
            for (int j = 0; j < MI; ++j) {
                hi[j] = *reinterpret_cast<const u32x4*>(t[j] + k);
                lo[j] = *reinterpret_cast<const u32x4*>(t[j] + LC + k);
            }
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const u32x4 f = b_frag(ad, i, k);
#pragma unroll
                for (int j = 0; j < MI; ++j) acc[i][j] = mma_bf16(f, lo[j], mma_bf16(f, hi[j], acc[i][j]));
            }
        }
        return;
    }
    // several slots, one after the other: each on the rows' pieces that it reaches into
    const bf16_t* t[MI];
    int mine[MI];
#pragma unroll
    for (int j = 0; j < MI; ++j) {
        t[j] = low_row(mw + 16 * j + l16) + 8 * quarter;
        mine[j] = slot_of(mw + 16 * j + l16);
    }
    const int last = slot_of(mw + 16 * MI - 1);
    for (int s = slot_of(mw); s <= last; ++s) {
        const int ad = adapter_of(a, s);
        if (ad < 0) continue;
        constexpr int NG = MI >= 4 || NI < 4 ? 2 : 4;               // pieces at a time
#pragma unroll
        for (int i0 = 0; i0 < NI; i0 += NG) {
            f32x4 sum[MI][NG];
#pragma unroll
            for (int j = 0; j < MI; ++j)
#pragma unroll
                for (int i = 0; i < NG; ++i) sum[j][i] = (f32x4){ 0.f, 0.f, 0.f, 0.f };
            for (int k = 0; k < LC; k += 32) {
                u32x4 f[NG];
#pragma unroll
                for (int i = 0; i < NG; ++i) f[i] = b_frag(ad, i0 + i, k);
#pragma unroll
                for (int j = 0; j < MI; ++j) {
                    const u32x4 hi = *reinterpret_cast<const u32x4*>(t[j] + k), lo = *reinterpret_cast<const u32x4*>(t[j] + LC + k);
#pragma unroll
                    for (int i = 0; i < NG; ++i) sum[j][i] = mma_bf16(f[i], lo, mma_bf16(f[i], hi, sum[j][i]));
                }
            }
#pragma unroll
            for (int j = 0; j < MI; ++j)
#pragma unroll
                for (int i = 0; i < NG; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i0 + i][j][r] += mine[j] == s ? sum[j][i][r] : 0.f;
        }
    }
}

// A wave's finished sums with bias and activation, in whole rows through LDS of its own (wbuf): acc[i][j][r] is (row 16 j + l16, weight row 16 i + 4 quarter + r).
// bias: of its weight rows; out_at: where its rows go (bytes from out0), all ones: nowhere; nc: the first column that it stores.
template <int MI, int NI, int KIND, int PASS, int PITCH, int CH>
__device__ __forceinline__ void store_wave_tile(const f32x4 (&acc)[NI][MI], const LinArgs& a, const float* bias, const uint32_t* out_at, char* out0, int nc, unsigned char* wbuf)
{
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
#pragma unroll
    for (int p = 0; p < MI * 16 / PASS; ++p) {
#pragma unroll
        for (int i = 0; i < NI; i += KIND == LIN_GLU ? 2 : 1) {
            const f32x4 b0 = *reinterpret_cast<const f32x4*>(bias + i * 16 + 4 * quarter);
            f32x4 b1 = b0;
            if constexpr (KIND == LIN_GLU) b1 = *reinterpret_cast<const f32x4*>(bias + (i + 1) * 16 + 4 * quarter);
#pragma unroll
            for (int jj = 0; jj < PASS / 16; ++jj) {
                const int j = p * (PASS / 16) + jj;
                __builtin_amdgcn_sched_barrier(0);  // (pieces computed far ahead of their stores would spill)
                f32x4 v = acc[i][j] + b0;
                if constexpr (KIND == LIN_GLU) {
                    const f32x4 u = acc[i + 1][j] + b1;
                    if (a.act == DRF_GLU_GELU)
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = glu(v[r], u[r], DRF_GLU_GELU);
                    else
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[r] = glu(v[r], u[r], DRF_GLU_SILU);
                }
                const bf16x4 o = { (bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3] };
                *reinterpret_cast<bf16x4*>(wbuf + (jj * 16 + l16) * PITCH + (KIND == LIN_GLU ? i / 2 : i) * 32 + quarter * 8) = o;
            }
        }
#pragma unroll 4
        for (int id = lane; id < PASS * CH; id += 64) {
            const int r = id / CH, c = id - r * CH, n = nc + c * 8;
            const uint32_t at = out_at[p * PASS + r];
            const u32x4 v = *reinterpret_cast<const u32x4*>(wbuf + r * PITCH + c * 16);
            if (at == 0xffffffffu || n >= a.N) continue;
            bf16_t* o = reinterpret_cast<bf16_t*>(out0 + at) + n;
            if (a.out_vec && n + 8 <= a.N) *reinterpret_cast<u32x4*>(o) = v;
            else {
                const bf16x8 e = __builtin_bit_cast(bf16x8, v);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (n + k < a.N) o[k] = e[k];
            }
        }
    }
}

}  // namespace

// The tiles of linear_tile.h, and the forms for few rows of linear_direct.h (8 to 64 of them a workgroup), by KIND (one file each).
template <int KIND> drf_status launch_linear_tile(int tile, const LinArgs& a, hipStream_t st);
template <typename T, int KIND> drf_status launch_linear_direct(int form, const LinArgs& a, hipStream_t st);

}  // namespace drf
