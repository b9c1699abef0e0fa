// Products of few rows, bf16 and fp32: operands straight from memory to registers, the inner axis dealt over the waves of a workgroup, 128 bytes of it at a time, which
// add up through LDS.  Such a launch is one chain of round trips to memory, and what counts is how many of the weights' bytes are asked for at once: every wave has its
// operands of U turns on the way.  One row, weights in the last-level cache: 1152 x 2 x 4608 with the activation 9.1 us (21 MB), 4608 x 1152 5.2 us (10.6 MB, on 8 by 8);
// 64 x 1152 x 6912, weights cold, 9.3 us; with 24 adapters of rank 16 among its rows, warm, 12.2.
#pragma once
#include "linear_device.h"

namespace drf {

namespace {

// c += w . x over 64 bytes of the inner axis, a lane's 16 each
__device__ inline f32x4 mma(const u32x4& w, const u32x4& x, f32x4 c, bf16_t) { return mma_bf16(w, x, c); }
__device__ inline f32x4 mma(const u32x4& w, const u32x4& x, f32x4 c, float)
{
    const f32x4 a = __builtin_bit_cast(f32x4, w), b = __builtin_bit_cast(f32x4, x);
#pragma unroll
    for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[k], b[k], c, 0, 0, 0);
    return c;
}

// 16 bytes from element k of a row of n on, at any address of an element; zeros behind the row's end
template <typename T> __device__ inline u32x4 load_row16(const T* row, int k, int n)
{
    constexpr int E = 16 / sizeof(T);
    typedef T piece __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    if (k + E <= n) return __builtin_bit_cast(u32x4, *reinterpret_cast<const piece*>(row + k));
    u32x4 z = { 0, 0, 0, 0 };
    if (k < n) {
        T v[E];
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = k + j < n ? row[k + j] : (T)0.f;
        __builtin_memcpy(&z, v, 16);
    }
    return z;
}

// The same in two parts, for rows of at least 16 bytes: a load that asks nothing (16 bytes that lie in the row, the last ones where k is near its end), so that many go out
// one behind the other, and what they are once they are there.
template <typename T> __device__ inline u32x4 load_near(const T* row, int k, int n)
{
    constexpr int E = 16 / sizeof(T);
    typedef T piece __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    return __builtin_bit_cast(u32x4, *reinterpret_cast<const piece*>(row + (k + E <= n ? k : n - E)));
}
__device__ inline u32x4 row_piece(u32x4 v, int k, int n, bf16_t) { return k < n ? v : (u32x4){ 0, 0, 0, 0 }; }     // (n is a multiple of 8)
__device__ inline u32x4 row_piece(u32x4 v, int k, int n, float)
{
    const int c = n - k;
    u32x4 r;
    r[0] = c >= 4 ? v[0] : c == 3 ? v[1] : c == 2 ? v[2] : c == 1 ? v[3] : 0u;
    r[1] = c >= 4 ? v[1] : c == 3 ? v[2] : c == 2 ? v[3] : 0u;
    r[2] = c >= 4 ? v[2] : c == 3 ? v[3] : 0u;
    r[3] = c >= 4 ? v[3] : 0u;
    return r;
}

struct Nothing { __device__ void operator()() const {} };

// acc += w x^T over a wave's share of the inner axis: turns of SP times 128 bytes, wave, wave + NW, .., U of them on the way; a lane's is `part` of its turn's.
// beside(): other loads, behind the first of these.
template <typename T, int MI, int NI, int NW, int U, int SP = 1, typename F = Nothing>
__device__ __forceinline__ void direct_product(f32x4 (&acc)[NI][MI], const T* const (&x)[MI], const T* const (&w)[NI], int K, int wave, int quarter, int part = 0, F beside = F{})
{
    constexpr int E = 16 / sizeof(T), CHUNK = 8 * E * SP, TURN = NW * CHUNK;
    const int first = wave * CHUNK, turns = first < K ? (K - first + TURN - 1) / TURN : 0;
    u32x4 fx[U][2][MI], fw[U][2][NI];
    auto load = [&](int t, int turn) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = first + turn * TURN + (8 * part + 4 * h + quarter) * E;
#pragma unroll
            for (int i = 0; i < NI; ++i) fw[t][h][i] = load_near(w[i], k, K);
#pragma unroll
            for (int j = 0; j < MI; ++j) fx[t][h][j] = load_near(x[j], k, K);
        }
    };
    auto multiply = [&](int t, int turn) __attribute__((always_inline)) {
        if (first + turn * TURN + CHUNK > K) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = first + turn * TURN + (8 * part + 4 * h + quarter) * E;
#pragma unroll
                for (int i = 0; i < NI; ++i) fw[t][h][i] = row_piece(fw[t][h][i], k, K, T{});
#pragma unroll
                for (int j = 0; j < MI; ++j) fx[t][h][j] = row_piece(fx[t][h][j], k, K, T{});
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int j = 0; j < MI; ++j) acc[i][j] = mma(fw[t][h][i], fx[t][h][j], acc[i][j], T{});
    };
#pragma unroll
    for (int t = 0; t < U; ++t)
        if (t < turns) load(t, t);
    beside();
    int it = 0;
    for (; it + 2 * U <= turns; it += U)            // (no questions between the loads: they are counted, and none waits for all)
#pragma unroll
        for (int t = 0; t < U; ++t) { multiply(t, it + t); load(t, it + t + U); }
    for (; it < turns; it += U)
#pragma unroll
        for (int t = 0; t < U; ++t) {
            if (it + t < turns) multiply(t, it + t);
            if (it + t + U < turns) load(t, it + t + U);
        }
}

// The adapter's part of four columns from n on of a row: x A^T of it times B's rows.
template <typename T> __device__ inline void add_low(f32x4& v, const LinArgs& a, int slot, int token, int n)
{
    const int ad = adapter_of(a, slot);
    if (ad < 0) return;
    const T* b[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) b[r] = (const T*)a.b + ((size_t)ad * a.N + (n + r < a.N ? n + r : a.N - 1)) * a.rank;
    const size_t row = (size_t)slot * a.tokens + token;
    constexpr int E = 16 / sizeof(T);
    for (int k = 0; k < a.rank; k += E) {
        float t[E];
        if constexpr (sizeof(T) == 2) {
            const bf16_t* p = (const bf16_t*)a.low + row * 2 * a.low_cols + k;
            const bf16x8 hi = *reinterpret_cast<const bf16x8*>(p), lo = *reinterpret_cast<const bf16x8*>(p + a.low_cols);
#pragma unroll
            for (int e = 0; e < E; ++e) t[e] = (float)hi[e] + (float)lo[e];
        } else {
            const f32x4 q = __builtin_bit_cast(f32x4, load_row16((const float*)a.low + row * a.low_cols, k, a.rank));
#pragma unroll
            for (int e = 0; e < E; ++e) t[e] = q[e];
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            T f[E];
            const u32x4 q = load_row16(b[r], k, a.rank);
            __builtin_memcpy(f, &q, 16);
#pragma unroll
            for (int e = 0; e < E; ++e) v[r] = fmaf(t[e], (float)f[e], v[r]);
        }
    }
}

// LANES MI rows by LANES NI rows of the weights (LIN_GLU: NI / 2 pairs of gates and values), LANES = 16 / SP.  SP > 1: a matrix instruction's sixteen rows are SP parts of the
// inner axis of LANES rows, of both operands; what counts of its result are the SP blocks on the diagonal, and a result's blocks are added up with the waves'.  So more
// workgroups share few weight rows.
template <typename T, int KIND, int MI, int NI, int NW, int U, int SP>
__global__ void __launch_bounds__(NW * 64) linear_direct_kernel(const LinArgs a)
{
    static_assert(KIND != LIN_GLU || NI % 2 == 0, "gates and values");
    static_assert(NW * MI * NI <= 64, "partial sums in 64 KB");
    __shared__ f32x4 part[NW][MI * NI][64];
    const int lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long id = a.first + blockIdx.x;
    constexpr int LANES = 16 / SP;
    const int lrow = l16 % LANES, half = l16 / LANES;
    const int tm = (int)(id / a.tiles_n), tn = (int)(id - (long long)tm * a.tiles_n), row0 = tm * LANES * MI;
    const int n0 = tn * (KIND == LIN_GLU ? LANES / 2 * NI : LANES * NI);
    const T *x[MI], *w[NI];
#pragma unroll
    for (int j = 0; j < MI; ++j) {                  // (rows behind a length are read and multiplied like others; what is not there is some row that is.  Neither is stored)
        int slot, token;
        locate_row(a, 0, row0 + LANES * j + lrow, slot, token);
        if (row0 + LANES * j + lrow >= a.slot_rows) slot = token = 0;
        x[j] = (const T*)a.x.data + slot * a.x.slot_stride + token * a.x.token_stride;
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        int n = KIND == LIN_GLU ? n0 + i / 2 * LANES + lrow : n0 + LANES * i + lrow;
        n = n < a.N ? n : a.N - 1;
        w[i] = (const T*)a.w + ((size_t)n + (KIND == LIN_GLU && i % 2 ? a.N : 0)) * a.K;
    }
    f32x4 acc[NI][MI];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < MI; ++j) acc[i][j] = (f32x4){ 0.f, 0.f, 0.f, 0.f };
    // results of 16 x 16, one for each of the first waves: lane (l16, quarter) has columns 4 quarter .. + 3 of row l16.  Its bias is asked for beside the product's operands
    // (feed-forward of 1 x 1152 x 4608: 17.2 -> 16.3 us; an adapter's operands asked for there as well took 64 x 1152 x 6912 of rank 16 from 16.4 to 17.0 us).
    constexpr int OUT = KIND == LIN_GLU ? NI / 2 : NI;
    static_assert(OUT * MI <= NW, "a result a wave");
    const int i = wave / MI, j = wave - i * MI, n = n0 + LANES * i + 4 * quarter, row = row0 + LANES * j + l16;
    float bias[KIND == LIN_GLU ? 2 : 1][4] = {};
    direct_product<T, MI, NI, NW, U, SP>(acc, x, w, a.K, wave, quarter, half, [&]() __attribute__((always_inline)) {
        if (!a.bias || wave >= OUT * MI) return;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int c = n + r < a.N ? n + r : a.N - 1;
            bias[0][r] = a.bias[c];
            if constexpr (KIND == LIN_GLU) bias[1][r] = a.bias[a.N + c];
        }
    });
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < MI; ++j) part[wave][i * MI + j][lane] = acc[i][j];
    __syncthreads();
    int sl, tk;
    if (wave < OUT * MI && (SP == 1 || (l16 < LANES && 4 * quarter < LANES)) && locate_row(a, 0, row, sl, tk) && n < a.N) {
        auto total = [&](int piece) {
            f32x4 v = part[0][piece * MI + j][lane];
#pragma unroll
            for (int u = 1; u < NW * SP; ++u) v += part[u / SP][piece * MI + j][lane + u % SP * (LANES / 4 * 16 + LANES)];
            return v;
        };
        f32x4 v = total(KIND == LIN_GLU ? 2 * i : i), u = v;
        if constexpr (KIND == LIN_GLU) u = total(2 * i + 1);
        if constexpr (KIND == LIN_ADAPT) add_low<T>(v, a, sl, tk, n);
        T* o = (T*)a.out.data + sl * a.out.slot_stride + tk * a.out.token_stride + n;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            v[r] += bias[0][r];
            if constexpr (KIND == LIN_GLU) v[r] = glu(v[r], u[r] + bias[1][r], a.act);
        }
        if (n + 4 <= a.N) {
            typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
            *reinterpret_cast<four*>(o) = (four){ (T)v[0], (T)v[1], (T)v[2], (T)v[3] };
        } else
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (n + r < a.N) o[r] = (T)v[r];
    }
}

template <typename T, int KIND, int MI, int NI, int NW, int U, int SP = 1> drf_status launch_direct_shape(LinArgs a, hipStream_t st)
{
    a.slot_rows = a.slots * a.tokens;
    constexpr int rows = 16 / SP * MI, columns = 16 / SP * NI / (KIND == LIN_GLU ? 2 : 1);
    a.tiles_n = (a.N + columns - 1) / columns;
    a.tiles = (long long)((a.slot_rows + rows - 1) / rows) * a.tiles_n;
    const long long most = 1 << 21;                                 // (a launch holds fewer than 2^32 threads)
    for (a.first = 0; a.first < a.tiles; a.first += most) {
        hipLaunchKernelGGL((linear_direct_kernel<T, KIND, MI, NI, NW, U, SP>), dim3((unsigned)std::min(most, a.tiles - a.first)), dim3(NW * 64), 0, st, a);
        DRF_HIP(hipGetLastError());
    }
    return DRF_OK;
}

}  // namespace

}  // namespace drf
