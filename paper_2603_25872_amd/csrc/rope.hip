// Rotary positions with several axes, and norms of queries and keys with the rotation in the same pass.
//
// One kernel for both: with n = (x - mean) / sqrt(var + eps) (or its simpler forms), p(c) the other column of c's pair and C, S its
// cosine and signed sine,
//   y_c = (n_c g_c + b_c) C_c + (n_p g_p + b_p) S_c = n_c A_c + n_p B_c + D_c,    A_c = g_c C_c, B_c = g_p S_c, D_c = b_c C_c + b_p S_c,
// so gains, biases, the scale of the queries and the angles come together in two or three numbers a column, which a lane forms once for its
// token and its columns and holds in registers over the token's heads.  A column that does not turn is n_c A_c + D_c alone: nothing times
// zero, so that an infinity in it, or in a column beside it, stays where it is.  The angles of a workgroup's tokens are formed once, by all its threads
// (in double precision: a position far from zero keeps its fraction of a turn), while the first heads are on their way.  What is left is a copy
// with a sum over a head's columns and two multiply-adds a column: bound by memory.
#include <algorithm>
#include <type_traits>

#include "common.h"

namespace drf {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxD = 128, kMaxPairs = kMaxD / 2, kThreads = 256, kWaves = kThreads / 64;

// The rotation as the kernels take it.
struct Pair { double turns; int axis, first; };     // per unit of position, in whole turns; its axis and the lower of its columns
struct Turns {
    Pair rec[kMaxPairs];
    uint8_t pair[kMaxD], other[kMaxD];      // the pair of a column that turns, and the other column of it (itself where nothing turns)
    double origin[DRF_ROPE_AXES], step[DRF_ROPE_AXES];
    int below[DRF_ROPE_AXES];               // tokens per unit of an axis
    int pairs, columns, n_axes;             // columns: those that turn
    const float* positions;                 // or NULL: the grid
    size_t slot_stride;
};

struct Side {                               // the queries or the keys
    const void* x; void* y;
    int64_t xs, xt, xh, ys, yt, yh;
    int heads;
    const float *gain, *bias;
    float scale;
};

struct HeadsArgs {
    Side q, k;
    int slots, tokens, d;
    const int32_t* lens;
    float eps;
    int tile, tiles, parts, head_waves;     // tokens a workgroup; its waves, head_waves of them over the heads, times `parts` workgroups
    int first;                              // workgroup that this launch begins with
    Turns r;
};

// position of token n of a slot on axis `axis`
__device__ inline double position(const Turns& r, int slot, int n, int axis)
{
    if (r.positions) return (double)r.positions[(size_t)slot * r.slot_stride + (size_t)n * r.n_axes + axis];
    double p = 0.0;
#pragma unroll
    for (int a = 0; a < DRF_ROPE_AXES; ++a) {                       // (all axes, so that nothing waits for a table entry to know which)
        if (a >= r.n_axes) break;
        const int at = n / r.below[a];
        n -= at * r.below[a];
        const double x = fma(r.step[a], (double)at, r.origin[a]);
        p = a == axis ? x : p;
    }
    return p;
}

// cos and sin of a turn of p units of position.  The angle is in double precision until a quarter turn at most is left of it, whose rounding to a float is
// in proportion to a sine or cosine that is small (of half a turn it is as large where a sine is near zero as elsewhere).
__device__ inline void turn(double p, double turns, float* c, float* s)
{
    p *= turns;
    p = 4.0 * (p - rint(p));
    const double quarter = rint(p);                                 // -2 .. 2
    float c0, s0;
    sincospif(0.5f * (float)(p - quarter), &s0, &c0);
    const int k = (int)quarter & 3;
    const float x = k & 1 ? s0 : c0, y = k & 1 ? c0 : s0;
    *c = k == 1 || k == 2 ? -x : x;
    *s = k >= 2 ? -y : y;
}

template <typename T> __device__ inline float to_f32(T v) { return (float)v; }

// Which columns a pair is of, and how the other ones of a lane's are read (a head's columns are read twice then, the second time from the near caches).
enum { ROPE_NO = 0, ROPE_IN_LANE = 1, ROPE_PIECE = 2, ROPE_HALF_PIECE = 3, ROPE_ELEMENT = 4 };

// A row (one head of one token) is P = d / E pieces of 16 bytes, one a lane, and a wave takes 64 / P tokens, so that all but the last few lanes
// work at any head width, and U heads of them at a time.  NORM: a drf_qk_norm.  Bound by memory: 4 slots x 16384 tokens x 16 heads of 72 in bf16
// turned, 302 MB, 68.5 us (4.4 TB/s, where a copy of 1 GiB reaches 5.05); q and k of 6 x 4096 x 16 of 72 with RMS norms, 226 MB, 53 us (4.3); the sums of
// four heads are formed beside one another (83 us with a head's shuffles behind the last one's).  One token: 3.9 us, a launch and three dependent reads.
constexpr int kHeads = 4;
template <typename T, int NORM, int ROPE>
__global__ void __launch_bounds__(kThreads) heads_kernel(const HeadsArgs a)
{
    constexpr int E = 16 / sizeof(T), U = kHeads;
    typedef T piece __attribute__((ext_vector_type(E)));
    typedef T half_piece __attribute__((ext_vector_type(E / 2)));
    extern __shared__ __attribute__((aligned(16))) float tab[];     // [token][pair](cos, sin)
    const int d = a.d, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // consecutive tiles on one XCD: they share the lines that a tile ends inside of
    int id = a.first + item_by_xcd(blockIdx.x, gridDim.x);
    const int part = id % a.parts;
    id /= a.parts;
    const int slot = id / a.tiles, t0 = (id - slot * a.tiles) * a.tile, left = slot_len(a.lens, slot, a.tokens) - t0;
    if (left <= 0) return;
    const int P = d / E, rpw = 64 / P, lr = lane / P, lp = lane - lr * P;
    const int tl = wave / a.head_waves * rpw + lr;                  // this lane's token of the tile
    const bool live = lr < rpw && tl < left;
    const int at = live ? tl : 0;                                   // (lanes without a row take part in the sums)
    const int col = lr < rpw ? lp * E : 0;
    // heads in chunks of U, the queries' and then the keys'; this wave's are c .. c1 - 1
    const int q_chunks = (a.q.heads + U - 1) / U, chunks = q_chunks + (a.k.heads + U - 1) / U, waves = a.parts * a.head_waves;
    const int w_id = part * a.head_waves + wave % a.head_waves, c1 = chunks * (w_id + 1) / waves;
    int ch = chunks * w_id / waves;

    // What the tables in the kernel's arguments and the norm's parameters give is asked for ahead of the heads: answers come in the order of the questions.
    const int first_pair = ROPE != ROPE_NO ? threadIdx.x % a.r.pairs : 0;
    Pair rec = a.r.rec[first_pair];
    int oc[E], pc[E];                                               // of this lane's columns: the others of their pairs, their pairs
#pragma unroll
    for (int j = 0; j < E; ++j) {
        oc[j] = ROPE == ROPE_IN_LANE ? col + (j ^ 1) : ROPE >= ROPE_PIECE ? a.r.other[col + j] : 0;
        pc[j] = ROPE == ROPE_IN_LANE ? (col + j) / 2 : ROPE >= ROPE_PIECE ? a.r.pair[col + j] : 0;
    }
    float g[E], go[E], b[E], bo[E];
    auto parameters = [&](const Side& e) {
#pragma unroll
        for (int j = 0; j < E; ++j) { g[j] = go[j] = 1.f; b[j] = bo[j] = 0.f; }
        if (NORM != DRF_QK_NONE && e.gain) {
#pragma unroll
            for (int j = 0; j < E; ++j) { g[j] = e.gain[col + j]; go[j] = e.gain[oc[j]]; }
        }
        if (NORM == DRF_QK_LAYER && e.bias) {
#pragma unroll
            for (int j = 0; j < E; ++j) { b[j] = e.bias[col + j]; bo[j] = e.bias[oc[j]]; }
        }
    };
    if (ch < c1) parameters(ch >= q_chunks ? a.k : a.q);
    piece v[U], w[U];
    auto load = [&](int chunk) {
        const bool is_k = chunk >= q_chunks;
        const Side& e = is_k ? a.k : a.q;
        const int h0 = (is_k ? chunk - q_chunks : chunk) * U;
        const T* x = (const T*)e.x + slot * e.xs + (int64_t)(t0 + at) * e.xt + h0 * e.xh;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const T* xr = x + (h0 + u < e.heads ? u : 0) * e.xh;
            v[u] = *reinterpret_cast<const piece*>(xr + col);
            if constexpr (ROPE == ROPE_PIECE) {
                w[u] = *reinterpret_cast<const piece*>(xr + oc[0]);
            } else if constexpr (ROPE == ROPE_HALF_PIECE) {
                const half_piece lo = *reinterpret_cast<const half_piece*>(xr + oc[0]), hi = *reinterpret_cast<const half_piece*>(xr + oc[E / 2]);
#pragma unroll
                for (int j = 0; j < E / 2; ++j) { w[u][j] = lo[j]; w[u][j + E / 2] = hi[j]; }
            } else if constexpr (ROPE == ROPE_ELEMENT) {
#pragma unroll
                for (int j = 0; j < E; ++j) w[u][j] = xr[oc[j]];
            }
        }
    };
    if (ch < c1) load(ch);
    if constexpr (ROPE != ROPE_NO) {
        const int nt = left < a.tile ? left : a.tile;
        for (int i = threadIdx.x; i < nt * a.r.pairs; i += kThreads) {
            const int n = i / a.r.pairs;
            if (i >= kThreads) rec = a.r.rec[i - n * a.r.pairs];
            turn(position(a.r, slot, t0 + n, rec.axis), rec.turns, &tab[2 * i], &tab[2 * i + 1]);
        }
        __syncthreads();
    }
    // sums over a row's lanes, of U rows at once
    auto row_sums = [&](float (&t)[U]) {
        for (int o = 1; o < P; o <<= 1) {
            float r[U];
#pragma unroll
            for (int u = 0; u < U; ++u) r[u] = __shfl_down(t[u], o, 64);
#pragma unroll
            for (int u = 0; u < U; ++u) t[u] += lp + o < P ? r[u] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) t[u] = __shfl(t[u], lr * P, 64);
    };
    const float inv_d = 1.f / (float)d;
    const int turning = a.r.columns - col;                          // of this lane's columns: the first so many turn
    float ka[E], kb[E], kd[E];
    int have = -1;                                                  // the side that they are for
    for (; ch < c1; ++ch) {
        const bool is_k = ch >= q_chunks;
        const Side& e = is_k ? a.k : a.q;
        if (have != (int)is_k) {
            if (have >= 0) parameters(e);
            have = is_k;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                float c = 1.f, s = 0.f;
                if (ROPE != ROPE_NO && j < turning) {
                    c = tab[2 * (at * a.r.pairs + pc[j])];
                    s = tab[2 * (at * a.r.pairs + pc[j]) + 1];
                    if (ROPE == ROPE_IN_LANE ? j % 2 == 0 : oc[j] > col + j) s = -s;    // (the first of a pair is the lower)
                }
                ka[j] = g[j] * e.scale * c; kb[j] = go[j] * e.scale * s;
                if constexpr (NORM == DRF_QK_LAYER) kd[j] = (ROPE != ROPE_NO && j < turning ? b[j] * c + bo[j] * s : b[j]) * e.scale;
            }
        }
        const int h0 = (is_k ? ch - q_chunks : ch) * U;
        T* y = (T*)e.y + slot * e.ys + (int64_t)(t0 + at) * e.yt + h0 * e.yh + col;
        float mean[U], inv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) { mean[u] = 0.f; inv[u] = 1.f; }
        if constexpr (NORM == DRF_QK_LAYER) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < E; ++j) mean[u] += to_f32(v[u][j]);
            row_sums(mean);
#pragma unroll
            for (int u = 0; u < U; ++u) mean[u] *= inv_d;
        }
        if constexpr (NORM != DRF_QK_NONE) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float t = 0.f;
#pragma unroll
                for (int j = 0; j < E; ++j) t = fmaf(to_f32(v[u][j]) - mean[u], to_f32(v[u][j]) - mean[u], t);
                inv[u] = t;
            }
            row_sums(inv);
#pragma unroll
            for (int u = 0; u < U; ++u) inv[u] = 1.f / sqrtf(inv[u] * inv_d + a.eps);
        }
        if (live) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                piece out;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    float r = (to_f32(v[u][j]) - mean[u]) * ka[j];
                    if constexpr (ROPE != ROPE_NO) {
                        const float turned = fmaf(to_f32(ROPE == ROPE_IN_LANE ? v[u][j ^ 1] : w[u][j]) - mean[u], kb[j], r);
                        r = j < turning ? turned : r;
                    }
                    if constexpr (NORM == DRF_QK_LAYER) r = fmaf(r, inv[u], kd[j]);
                    else if constexpr (NORM == DRF_QK_RMS) r *= inv[u];
                    out[j] = (T)r;
                }
                if (h0 + u < e.heads) *reinterpret_cast<piece*>(y + u * e.yh) = out;
            }
        }
        if (ch + 1 < c1) load(ch + 1);
    }
}

// Any width, stride and alignment: a wave a row, a column or two a lane, angles by every lane for itself.
template <typename T, int NORM>
__global__ void __launch_bounds__(kThreads) heads_any_kernel(const HeadsArgs a, long long rows)
{
    const int lane = threadIdx.x & 63, d = a.d, all = a.q.heads + a.k.heads;
    for (long long row = (long long)blockIdx.x * kWaves + (threadIdx.x >> 6); row < rows; row += (long long)gridDim.x * kWaves) {
        const int hh = (int)(row % all);
        const long long sn = row / all;
        const int slot = (int)(sn / a.tokens), n = (int)(sn % a.tokens), w = hh >= a.q.heads, h = w ? hh - a.q.heads : hh;
        if (n >= slot_len(a.lens, slot, a.tokens)) continue;
        const Side& e = w ? a.k : a.q;
        const T* x = (const T*)e.x + slot * e.xs + (int64_t)n * e.xt + h * e.xh;
        T* y = (T*)e.y + slot * e.ys + (int64_t)n * e.yt + h * e.yh;
        auto wave_sum = [](float v) {
#pragma unroll
            for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, 64);
            return v;
        };
        float v[2], o[2];
        int oc[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int c = lane + 64 * j;
            oc[j] = c < d ? (c < a.r.columns ? a.r.other[c] : c) : 0;
            v[j] = c < d ? to_f32(x[c]) : 0.f;
            o[j] = c < d ? to_f32(x[oc[j]]) : 0.f;
        }
        float mean = 0.f, inv = 1.f;
        if constexpr (NORM == DRF_QK_LAYER) mean = wave_sum(v[0] + v[1]) / (float)d;
        if constexpr (NORM != DRF_QK_NONE) {
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < 2; ++j) s += lane + 64 * j < d ? (v[j] - mean) * (v[j] - mean) : 0.f;
            inv = 1.f / sqrtf(wave_sum(s) / (float)d + a.eps);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int c = lane + 64 * j;
            if (c >= d) continue;
            auto affine = [&](float z, int col) {
                z = (z - mean) * inv;
                if (e.gain) z *= e.gain[col];
                if (e.bias) z += e.bias[col];
                return z * e.scale;
            };
            float r = affine(v[j], c);
            if (c < a.r.columns) {
                const Pair& p = a.r.rec[a.r.pair[c]];
                float cs, sn_;
                turn(position(a.r, slot, n, p.axis), p.turns, &cs, &sn_);
                const float z = affine(o[j], oc[j]);
                r = p.first == c ? fmaf(r, cs, -z * sn_) : fmaf(r, cs, z * sn_);
            }
            y[c] = (T)r;
        }
    }
}

drf_status fill_turns(const drf_rope_config* rc, int head_dim, const float* positions, size_t slot_stride, Turns* t)
{
    *t = Turns{};
    if (!rc) return DRF_OK;
    if (rc->n_axes < 1 || rc->n_axes > DRF_ROPE_AXES) DRF_FAIL(DRF_EINVAL, "n_axes %d outside 1..%d", rc->n_axes, DRF_ROPE_AXES);
    if (!(rc->theta > 0.0) || !std::isfinite(rc->theta)) DRF_FAIL(DRF_EINVAL, "theta must be a positive number");
    if (rc->layout != DRF_ROPE_PAIRS && rc->layout != DRF_ROPE_HALVES) DRF_FAIL(DRF_EINVAL, "unknown rope layout");
    long long below = 1;
    for (int a = rc->n_axes - 1; a >= 0; --a) {
        if (rc->dim[a] < 0 || rc->dim[a] % 2) DRF_FAIL(DRF_EINVAL, "axis %d: dim %d is not an even number >= 0", a, rc->dim[a]);
        if (rc->extent[a] < 1) DRF_FAIL(DRF_EINVAL, "axis %d: extent must be >= 1", a);
        if (!std::isfinite(rc->origin[a]) || !std::isfinite(rc->step[a])) DRF_FAIL(DRF_EINVAL, "axis %d: origin and step must be finite", a);
        if (below > 0x7fffffffLL) below = 0x7fffffffLL;         // no token index gets there
        t->below[a] = (int)below;
        t->origin[a] = rc->origin[a]; t->step[a] = rc->step[a];
        below *= rc->extent[a];
    }
    int column = 0;
    for (int a = 0; a < rc->n_axes; ++a) {
        if (rc->dim[a] > head_dim - column) DRF_FAIL(DRF_ESHAPE, "the axes turn more columns than the %d of a head", head_dim);
        const int half = rc->dim[a] / 2;
        for (int i = 0; i < half; ++i) {
            const int p = t->pairs++;
            const bool pairs = rc->layout == DRF_ROPE_PAIRS;
            const int c0 = pairs ? column + 2 * i : column + i, c1 = pairs ? column + 2 * i + 1 : column + half + i;
            t->rec[p] = { std::pow(rc->theta, -2.0 * i / rc->dim[a]) / (2.0 * 3.14159265358979323846), a, c0 };
            t->other[c0] = (uint8_t)c1; t->other[c1] = (uint8_t)c0;
            t->pair[c0] = t->pair[c1] = (uint8_t)p;
        }
        column += rc->dim[a];
    }
    for (int c = column; c < head_dim; ++c) t->other[c] = (uint8_t)c;
    t->columns = column; t->n_axes = rc->n_axes;
    t->positions = positions; t->slot_stride = slot_stride;
    return DRF_OK;
}

drf_status fill_side(const char* what, const drf_heads* in, const drf_heads* out, int slots, int tokens, int heads, int head_dim, bool* vec, int unit, Side* s)
{
    if (!in || !out || !in->data || !out->data) DRF_FAIL(DRF_EINVAL, "%s: NULL tensor", what);
    const drf_heads x = used_strides(*in, slots, tokens, heads), y = used_strides(*out, slots, tokens, heads);
    if (x.data == y.data && (x.slot_stride != y.slot_stride || x.token_stride != y.token_stride || x.head_stride != y.head_stride))
        DRF_FAIL(DRF_EINVAL, "%s: input and output share an address but not their strides", what);
    if (rows_overlap(y, slots, tokens, heads, head_dim)) DRF_FAIL(DRF_EINVAL, "%s: rows of the output lie on one another", what);
    s->x = x.data; s->xs = x.slot_stride; s->xt = x.token_stride; s->xh = x.head_stride;
    s->y = y.data; s->ys = y.slot_stride; s->yt = y.token_stride; s->yh = y.head_stride;
    s->heads = heads;
    for (const drf_heads& t : { x, y })
        *vec = *vec && (reinterpret_cast<uintptr_t>(t.data) & 15u) == 0 && t.slot_stride % unit == 0 && t.token_stride % unit == 0 && t.head_stride % unit == 0;
    return DRF_OK;
}

template <typename T, int NORM> void go(const HeadsArgs& a, int rope, unsigned grid, hipStream_t st)
{
    const size_t lds = rope == ROPE_NO ? 0 : (size_t)a.tile * a.r.pairs * 2 * sizeof(float);
    switch (rope) {
    case ROPE_NO: hipLaunchKernelGGL((heads_kernel<T, NORM, ROPE_NO>), dim3(grid), dim3(kThreads), lds, st, a); break;
    case ROPE_IN_LANE: hipLaunchKernelGGL((heads_kernel<T, NORM, ROPE_IN_LANE>), dim3(grid), dim3(kThreads), lds, st, a); break;
    case ROPE_PIECE: hipLaunchKernelGGL((heads_kernel<T, NORM, ROPE_PIECE>), dim3(grid), dim3(kThreads), lds, st, a); break;
    case ROPE_HALF_PIECE: hipLaunchKernelGGL((heads_kernel<T, NORM, ROPE_HALF_PIECE>), dim3(grid), dim3(kThreads), lds, st, a); break;
    default: hipLaunchKernelGGL((heads_kernel<T, NORM, ROPE_ELEMENT>), dim3(grid), dim3(kThreads), lds, st, a);
    }
}

template <typename T> drf_status launch(HeadsArgs& a, int norm, int rope, bool vec, hipStream_t st)
{
    const int all = a.q.heads + a.k.heads;
    if (!vec) {
        const long long rows = (long long)a.slots * a.tokens * all, most = (rows + kWaves - 1) / kWaves, grid = most < 1 << 20 ? most : 1 << 20;
        if (norm == DRF_QK_NONE) hipLaunchKernelGGL((heads_any_kernel<T, DRF_QK_NONE>), dim3((unsigned)grid), dim3(kThreads), 0, st, a, rows);
        else if (norm == DRF_QK_RMS) hipLaunchKernelGGL((heads_any_kernel<T, DRF_QK_RMS>), dim3((unsigned)grid), dim3(kThreads), 0, st, a, rows);
        else hipLaunchKernelGGL((heads_any_kernel<T, DRF_QK_LAYER>), dim3((unsigned)grid), dim3(kThreads), 0, st, a, rows);
        DRF_HIP(hipGetLastError());
        return DRF_OK;
    }
    // A workgroup's waves share the tokens' angles: all four over the heads where there are that many chunks of them, the rest over more tokens.
    const int chunks = (a.q.heads + kHeads - 1) / kHeads + (a.k.heads + kHeads - 1) / kHeads;
    a.head_waves = chunks >= 4 ? 4 : chunks >= 2 ? 2 : 1;
    a.tile = kWaves / a.head_waves * (64 / (a.d * (int)sizeof(T) / 16));
    a.tiles = (a.tokens + a.tile - 1) / a.tile;
    const long long groups = (long long)a.tiles * a.slots;
    // and over several workgroups until there is one for every CU
    a.parts = 1;
    while (a.parts * 2 * a.head_waves <= chunks && groups * a.parts < 256) a.parts *= 2;
    const long long all_groups = groups * a.parts, most = 1 << 23;              // (a launch holds fewer than 2^32 threads)
    if (all_groups > 0x7fffffffLL) DRF_FAIL(DRF_ESHAPE, "more than 2^31 workgroups");
    for (long long first = 0; first < all_groups; first += most) {
        a.first = (int)first;
        const unsigned grid = (unsigned)(all_groups - first < most ? all_groups - first : most);
        if (norm == DRF_QK_NONE) go<T, DRF_QK_NONE>(a, rope, grid, st);
        else if (norm == DRF_QK_RMS) go<T, DRF_QK_RMS>(a, rope, grid, st);
        else go<T, DRF_QK_LAYER>(a, rope, grid, st);
        DRF_HIP(hipGetLastError());
    }
    return DRF_OK;
}

drf_status run_heads(HeadsArgs& a, const drf_rope_config* rope, drf_dtype dtype, int norm, bool vec, hipStream_t st)
{
    const int unit = dtype == DRF_BF16 ? 8 : 4;
    vec = vec && a.d % unit == 0;
    int kind = ROPE_NO;
    if (a.r.columns && rope->layout == DRF_ROPE_PAIRS) {
        kind = ROPE_IN_LANE;
    } else if (a.r.columns) {
        int granule = unit;                                         // columns that keep together in a pair's other half
        for (int i = 0; i < rope->n_axes; ++i)
            while (rope->dim[i] / 2 % granule) granule /= 2;
        kind = granule == unit ? ROPE_PIECE : dtype == DRF_BF16 && granule == unit / 2 ? ROPE_HALF_PIECE : ROPE_ELEMENT;
    }
    return dtype == DRF_BF16 ? launch<bf16_t>(a, norm, kind, vec, st) : launch<float>(a, norm, kind, vec, st);
}

drf_status check_sizes(drf_dtype dtype, int slots, int tokens, int heads, int head_dim)
{
    if (dtype != DRF_F32 && dtype != DRF_BF16) DRF_FAIL(DRF_EINVAL, "unknown dtype");
    if (slots < 0 || tokens < 0 || heads < 1 || head_dim < 1) DRF_FAIL(DRF_EINVAL, "slots and tokens must be >= 0, heads and head_dim >= 1");
    if (head_dim > kMaxD) DRF_FAIL(DRF_ESHAPE, "head_dim must be <= %d (got %d)", kMaxD, head_dim);
    if (heads > 65535) DRF_FAIL(DRF_ESHAPE, "more than 65535 heads");
    if (tokens > 1 << 30) DRF_FAIL(DRF_ESHAPE, "more than 2^30 tokens");
    return DRF_OK;
}

}  // namespace

}  // namespace drf

using namespace drf;

extern "C" drf_status drf_rope(const drf_rope_config* rope, drf_dtype dtype, int slots, int tokens, int heads, int head_dim,
                               const int32_t* lens, const float* positions, size_t positions_slot_stride, const drf_heads* x,
                               const drf_heads* out, void* hip_stream)
{
    drf_status rc = check_sizes(dtype, slots, tokens, heads, head_dim);
    if (rc != DRF_OK) return rc;
    if (!rope) DRF_FAIL(DRF_EINVAL, "rope is NULL");
    HeadsArgs a{};
    if ((rc = fill_turns(rope, head_dim, positions, positions_slot_stride, &a.r)) != DRF_OK) return rc;
    if (slots == 0 || tokens == 0) return DRF_OK;
    bool vec = true;
    if ((rc = fill_side("x", x, out, slots, tokens, heads, head_dim, &vec, dtype == DRF_BF16 ? 8 : 4, &a.q)) != DRF_OK) return rc;
    a.q.scale = 1.f;
    a.k = a.q; a.k.heads = 0;
    a.slots = slots; a.tokens = tokens; a.d = head_dim; a.lens = lens;
    return run_heads(a, rope, dtype, DRF_QK_NONE, vec, (hipStream_t)hip_stream);
}

extern "C" drf_status drf_qk_norm_rope(const drf_qk_config* cfg, const drf_rope_config* rope, const drf_attn_shape* shape,
                                       const float* positions, size_t positions_slot_stride, const drf_heads* q, const drf_heads* k,
                                       const drf_heads* q_out, const drf_heads* k_out, void* hip_stream)
{
    if (!cfg || !shape) DRF_FAIL(DRF_EINVAL, "NULL configuration");
    const drf_attn_shape& s = *shape;
    drf_status rc = check_sizes(s.dtype, s.slots, s.q_tokens, s.q_heads, s.head_dim);
    if (rc != DRF_OK) return rc;
    if ((rc = check_sizes(s.dtype, s.slots, s.kv_tokens, s.kv_heads, s.head_dim)) != DRF_OK) return rc;
    if (s.kv_tokens != s.q_tokens) DRF_FAIL(DRF_EINVAL, "q and k have %d and %d tokens", s.q_tokens, s.kv_tokens);
    if (s.kv_lens && s.kv_lens != s.q_lens) DRF_FAIL(DRF_EINVAL, "q and k have lengths of their own");
    if (cfg->norm != DRF_QK_NONE && cfg->norm != DRF_QK_RMS && cfg->norm != DRF_QK_LAYER) DRF_FAIL(DRF_EINVAL, "unknown norm");
    if (!(cfg->eps >= 0.0) || !std::isfinite(cfg->eps) || !std::isfinite(cfg->q_scale)) DRF_FAIL(DRF_EINVAL, "eps must be >= 0 and q_scale finite");
    if (cfg->norm == DRF_QK_NONE && (cfg->q_gain || cfg->k_gain)) DRF_FAIL(DRF_EINVAL, "gains without a norm");
    if (cfg->norm != DRF_QK_LAYER && (cfg->q_bias || cfg->k_bias)) DRF_FAIL(DRF_EINVAL, "biases belong to DRF_QK_LAYER");
    HeadsArgs a{};
    if ((rc = fill_turns(rope, s.head_dim, positions, positions_slot_stride, &a.r)) != DRF_OK) return rc;
    if (s.slots == 0 || s.q_tokens == 0) return DRF_OK;
    bool vec = true;
    const int unit = s.dtype == DRF_BF16 ? 8 : 4;
    if ((rc = fill_side("q", q, q_out, s.slots, s.q_tokens, s.q_heads, s.head_dim, &vec, unit, &a.q)) != DRF_OK) return rc;
    if ((rc = fill_side("k", k, k_out, s.slots, s.kv_tokens, s.kv_heads, s.head_dim, &vec, unit, &a.k)) != DRF_OK) return rc;
    a.q.scale = cfg->q_scale; a.k.scale = 1.f;
    a.q.gain = cfg->q_gain; a.q.bias = cfg->q_bias; a.k.gain = cfg->k_gain; a.k.bias = cfg->k_bias;
    a.slots = s.slots; a.tokens = s.q_tokens; a.d = s.head_dim; a.lens = s.q_lens;
    a.eps = cfg->eps > 0.0 ? std::max((float)cfg->eps, 1.17549435e-38f) : 0.f;     // (one that fp32 does not hold is still no zero: a row of zeros stays one)
    return run_heads(a, rope, s.dtype, cfg->norm, vec, (hipStream_t)hip_stream);
}
