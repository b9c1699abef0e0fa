// Rotary positions with several axes, and norms of queries and keys with the rotation in the same pass.
//
// One kernel for both: with n = (x - mean) / sqrt(var + eps) (or its simpler forms), p(c) the other column of c's pair and C, S its
// cosine and signed sine,
//   y_c = (n_c g_c + b_c) C_c + (n_p g_p + b_p) S_c = n_c A_c + n_p B_c + D_c,    A_c = g_c C_c, B_c = g_p S_c, D_c = b_c C_c + b_p S_c,
// so gains, biases, the scale of the queries and the angles of a token come together in a table of two or three numbers a column, which a
// workgroup forms once for its few tokens (angles in double precision: a position far from zero keeps its fraction of a turn) and uses for
// every head of them.  What is left is a copy with a sum over d columns and two multiply-adds a column: bound by memory.
#include <type_traits>

#include "common.h"

namespace drf {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxD = 128, kMaxPairs = kMaxD / 2, kThreads = 256, kWaves = kThreads / 64;

// The rotation as the kernels take it.
struct Turns {
    double turns[kMaxPairs];                // of pair i per unit of position, in whole turns
    uint8_t axis[kMaxPairs], first[kMaxPairs], second[kMaxPairs];       // its axis and its two columns
    uint8_t other[kMaxD];                   // the other column of a column's pair (itself where nothing turns)
    double origin[DRF_ROPE_AXES], step[DRF_ROPE_AXES];
    int below[DRF_ROPE_AXES], extent[DRF_ROPE_AXES];    // tokens per unit of an axis, its extent
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
    int tile, tiles, parts, per_part;       // tokens a workgroup; heads in `parts` ranges of per_part
    int heads_inner;                        // rows run over the heads of a token first
    int granule;                            // columns that keep together in a pair's other half (DRF_ROPE_HALVES)
    Turns r;
};

__device__ inline int slot_len(const int32_t* lens, int slot, int tokens)
{
    if (!lens) return tokens;
    const int n = lens[slot];
    return n < 0 ? 0 : n < tokens ? n : tokens;
}

// cos and sin of pair i at token n of a slot
__device__ inline void turn(const Turns& r, int slot, int n, int i, float* c, float* s)
{
    const int a = r.axis[i];
    double p;
    if (r.positions) {
        p = (double)r.positions[(size_t)slot * r.slot_stride + (size_t)n * r.n_axes + a];
    } else {
        int at = n / r.below[a];
        if (a > 0) at %= r.extent[a];
        p = fma(r.step[a], (double)at, r.origin[a]);
    }
    p *= r.turns[i];
    sincospif(2.f * (float)(p - rint(p)), s, c);
}

template <typename T> __device__ inline float to_f32(T v) { return (float)v; }

// Pieces of 16 bytes: a row (one head of one token) is P of them, one a lane, and a wave takes 64 / P rows at a time, so that all but the
// last few lanes work at any head width.  NORM: a drf_qk_norm; ROPE: 0 none, 1 pairs, 2 halves.
template <typename T, int NORM, int ROPE>
__global__ void __launch_bounds__(kThreads) heads_kernel(const HeadsArgs a)
{
    constexpr int E = 16 / sizeof(T), U = 2;
    typedef T piece __attribute__((ext_vector_type(E)));
    extern __shared__ __attribute__((aligned(16))) float tab[];     // [A, B, D][q, k][token][column]
    const int d = a.d, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int id = blockIdx.x;
    const int part = id % a.parts;
    id /= a.parts;
    const int slot = id / a.tiles, t0 = (id - slot * a.tiles) * a.tile;
    const int left = slot_len(a.lens, slot, a.tokens) - t0;
    if (left <= 0) return;
    const int nt = left < a.tile ? left : a.tile;
    const int all = a.q.heads + a.k.heads, h0 = part * a.per_part, h1 = h0 + a.per_part < all ? h0 + a.per_part : all, nh = h1 - h0;
    const int plane = 2 * a.tile * d;
    const int P = d / E, rpw = 64 / P, lr = lane / P, lp = lane - lr * P;

    // the table
    if constexpr (ROPE != 0) {
        for (int i = tid; i < nt * a.r.pairs; i += kThreads) {
            const int n = i / a.r.pairs, p = i - n * a.r.pairs, c0 = a.r.first[p], c1 = a.r.second[p];
            float c, s;
            turn(a.r, slot, t0 + n, p, &c, &s);
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const Side& e = w ? a.k : a.q;
                const float g0 = (e.gain ? e.gain[c0] : 1.f) * e.scale, g1 = (e.gain ? e.gain[c1] : 1.f) * e.scale;
                float* t = tab + (w * a.tile + n) * d;
                t[c0] = g0 * c; t[c1] = g1 * c;
                t[plane + c0] = -g1 * s; t[plane + c1] = g0 * s;
                if constexpr (NORM == DRF_QK_LAYER) {
                    const float b0 = e.bias ? e.bias[c0] * e.scale : 0.f, b1 = e.bias ? e.bias[c1] * e.scale : 0.f;
                    t[2 * plane + c0] = b0 * c - b1 * s; t[2 * plane + c1] = b0 * s + b1 * c;
                }
            }
        }
    }
    {
        const int from = ROPE != 0 ? a.r.columns : 0, rest = d - from;
        for (int i = tid; i < 2 * nt * rest; i += kThreads) {
            const int row = i / rest, c = from + i - row * rest, w = row >= nt, n = row - w * nt;
            const Side& e = w ? a.k : a.q;
            float* t = tab + (w * a.tile + n) * d + c;
            t[0] = (e.gain ? e.gain[c] : 1.f) * e.scale;
            t[plane] = 0.f;
            if constexpr (NORM == DRF_QK_LAYER) t[2 * plane] = e.bias ? e.bias[c] * e.scale : 0.f;
        }
    }
    __syncthreads();

    const int rows = nh * nt, inner = a.heads_inner ? nh : nt;
    // sum over a row's lanes
    auto row_sum = [&](float v) {
        for (int o = 1; o < P; o <<= 1) {
            const float u = __shfl_down(v, o, 64);
            v += lp + o < P ? u : 0.f;
        }
        return __shfl(v, lr * P, 64);
    };
    for (int base = wave * rpw * U; base < rows; base += kWaves * rpw * U) {
        piece x[U], xo[U];
        T* y[U];
        const float* t[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = base + u * rpw + lr;
            y[u] = nullptr;
            if (lr < rpw && row < rows) {
                const int o = row / inner, i = row - o * inner;
                const int n = a.heads_inner ? o : i, hh = h0 + (a.heads_inner ? i : o), w = hh >= a.q.heads;
                const Side& e = w ? a.k : a.q;
                const int h = w ? hh - a.q.heads : hh;
                const T* xr = (const T*)e.x + slot * e.xs + (int64_t)(t0 + n) * e.xt + h * e.xh;
                x[u] = *reinterpret_cast<const piece*>(xr + lp * E);
                if constexpr (ROPE == 2) {
                    if (a.granule == E) {
                        xo[u] = *reinterpret_cast<const piece*>(xr + a.r.other[lp * E]);
                    } else if (E == 8 && a.granule == E / 2) {
                        typedef T half_piece __attribute__((ext_vector_type(E / 2)));
                        const half_piece lo = *reinterpret_cast<const half_piece*>(xr + a.r.other[lp * E]);
                        const half_piece hi = *reinterpret_cast<const half_piece*>(xr + a.r.other[lp * E + E / 2]);
#pragma unroll
                        for (int j = 0; j < E / 2; ++j) { xo[u][j] = lo[j]; xo[u][j + E / 2] = hi[j]; }
                    } else {
#pragma unroll
                        for (int j = 0; j < E; ++j) xo[u][j] = xr[a.r.other[lp * E + j]];
                    }
                }
                y[u] = (T*)e.y + slot * e.ys + (int64_t)(t0 + n) * e.yt + h * e.yh + lp * E;
                t[u] = tab + (w * a.tile + n) * d + lp * E;
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j) x[u][j] = (T)0.f;
                if constexpr (ROPE == 2) xo[u] = x[u];
                t[u] = tab;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[E], o[E];
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] = to_f32(x[u][j]);
            float mean = 0.f, inv = 1.f;
            if constexpr (NORM == DRF_QK_LAYER) {
                float s = 0.f;
#pragma unroll
                for (int j = 0; j < E; ++j) s += v[j];
                mean = row_sum(s) / (float)d;
#pragma unroll
                for (int j = 0; j < E; ++j) v[j] -= mean;
            }
            if constexpr (NORM != DRF_QK_NONE) {
                float s = 0.f;
#pragma unroll
                for (int j = 0; j < E; ++j) s = fmaf(v[j], v[j], s);
                inv = 1.f / sqrtf(row_sum(s) / (float)d + a.eps);
            }
            if constexpr (ROPE == 1) {
#pragma unroll
                for (int j = 0; j < E; ++j) o[j] = v[j ^ 1];
            } else if constexpr (ROPE == 2) {
#pragma unroll
                for (int j = 0; j < E; ++j) o[j] = to_f32(xo[u][j]) - mean;
            }
            if (y[u]) {
                piece out;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    float r = v[j] * inv * t[u][j];
                    if constexpr (ROPE != 0) r = fmaf(o[j] * inv, t[u][plane + j], r);
                    if constexpr (NORM == DRF_QK_LAYER) r += t[u][2 * plane + j];
                    out[j] = (T)r;
                }
                *reinterpret_cast<piece*>(y[u]) = out;
            }
        }
    }
}

// Any width, stride and alignment: a wave a row, a column or two a lane, angles by every lane for itself.
template <typename T, int NORM>
__global__ void __launch_bounds__(kThreads) heads_any_kernel(const HeadsArgs a, long long rows)
{
    const int lane = threadIdx.x & 63, d = a.d, all = a.q.heads + a.k.heads;
    const long long row = (long long)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (row >= rows) return;
    const int hh = (int)(row % all);
    const long long sn = row / all;
    const int slot = (int)(sn / a.tokens), n = (int)(sn % a.tokens), w = hh >= a.q.heads, h = w ? hh - a.q.heads : hh;
    if (n >= slot_len(a.lens, slot, a.tokens)) return;
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
            int i = 0;                          // the pair that column c belongs to
            while (a.r.first[i] != c && a.r.second[i] != c) ++i;
            float cs, sn_;
            turn(a.r, slot, n, i, &cs, &sn_);
            const float z = affine(o[j], oc[j]);
            r = a.r.first[i] == c ? fmaf(r, cs, -z * sn_) : fmaf(r, cs, z * sn_);
        }
        y[c] = (T)r;
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
        t->below[a] = (int)below; t->extent[a] = rc->extent[a];
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
            t->axis[p] = (uint8_t)a;
            t->first[p] = (uint8_t)(pairs ? column + 2 * i : column + i);
            t->second[p] = (uint8_t)(pairs ? column + 2 * i + 1 : column + half + i);
            t->other[t->first[p]] = t->second[p]; t->other[t->second[p]] = t->first[p];
            t->turns[p] = std::pow(rc->theta, -2.0 * i / rc->dim[a]) / (2.0 * 3.14159265358979323846);
        }
        column += rc->dim[a];
    }
    for (int c = column; c < head_dim; ++c) t->other[c] = (uint8_t)c;
    t->columns = column; t->n_axes = rc->n_axes;
    t->positions = positions; t->slot_stride = slot_stride;
    return DRF_OK;
}

drf_status fill_side(const char* what, const drf_heads* x, const drf_heads* y, int heads, bool* vec, int unit, Side* s)
{
    if (!x || !y || !x->data || !y->data) DRF_FAIL(DRF_EINVAL, "%s: NULL tensor", what);
    if (x->data == y->data && (x->slot_stride != y->slot_stride || x->token_stride != y->token_stride || x->head_stride != y->head_stride))
        DRF_FAIL(DRF_EINVAL, "%s: input and output share an address but not their strides", what);
    s->x = x->data; s->xs = x->slot_stride; s->xt = x->token_stride; s->xh = x->head_stride;
    s->y = y->data; s->ys = y->slot_stride; s->yt = y->token_stride; s->yh = y->head_stride;
    s->heads = heads;
    for (const drf_heads* t : { x, y })
        *vec = *vec && (reinterpret_cast<uintptr_t>(t->data) & 15u) == 0 && t->slot_stride % unit == 0 && t->token_stride % unit == 0 && t->head_stride % unit == 0;
    return DRF_OK;
}

template <typename T, int NORM, int ROPE> void go(const HeadsArgs& a, unsigned grid, size_t lds, hipStream_t st)
{
    hipLaunchKernelGGL((heads_kernel<T, NORM, ROPE>), dim3(grid), dim3(kThreads), lds, st, a);
}

template <typename T> drf_status launch(HeadsArgs& a, int norm, int rope, bool vec, hipStream_t st)
{
    const int all = a.q.heads + a.k.heads;
    if (!vec) {
        const long long rows = (long long)a.slots * a.tokens * all, grid = (rows + kWaves - 1) / kWaves;
        if (grid > 0x7fffffLL) DRF_FAIL(DRF_ESHAPE, "too many unaligned rows");
        if (norm == DRF_QK_NONE) hipLaunchKernelGGL((heads_any_kernel<T, DRF_QK_NONE>), dim3((unsigned)grid), dim3(kThreads), 0, st, a, rows);
        else if (norm == DRF_QK_RMS) hipLaunchKernelGGL((heads_any_kernel<T, DRF_QK_RMS>), dim3((unsigned)grid), dim3(kThreads), 0, st, a, rows);
        else hipLaunchKernelGGL((heads_any_kernel<T, DRF_QK_LAYER>), dim3((unsigned)grid), dim3(kThreads), 0, st, a, rows);
        DRF_HIP(hipGetLastError());
        return DRF_OK;
    }
    a.tile = 8;
    a.tiles = (a.tokens + a.tile - 1) / a.tile;
    const long long groups = (long long)a.tiles * a.slots;
    a.parts = 1;
    while (a.parts < all && groups * a.parts < 1024) a.parts *= 2;
    if (a.parts > all) a.parts = all;
    a.per_part = (all + a.parts - 1) / a.parts;
    a.parts = (all + a.per_part - 1) / a.per_part;
    if (groups * a.parts > 0x7fffffLL) DRF_FAIL(DRF_ESHAPE, "too many tokens");
    // rows in the order that the memory of a token tile has
    a.heads_inner = llabs(a.q.xh) < llabs(a.q.xt);
    const size_t lds = (size_t)(norm == DRF_QK_LAYER ? 3 : 2) * 2 * a.tile * a.d * sizeof(float);
    const unsigned grid = (unsigned)(groups * a.parts);
#define DRF_GO(N) (rope == 0 ? go<T, N, 0>(a, grid, lds, st) : rope == 1 ? go<T, N, 1>(a, grid, lds, st) : go<T, N, 2>(a, grid, lds, st))
    if (norm == DRF_QK_NONE) DRF_GO(DRF_QK_NONE);
    else if (norm == DRF_QK_RMS) DRF_GO(DRF_QK_RMS);
    else DRF_GO(DRF_QK_LAYER);
#undef DRF_GO
    DRF_HIP(hipGetLastError());
    return DRF_OK;
}

drf_status run_heads(HeadsArgs& a, const drf_rope_config* rope, drf_dtype dtype, int norm, bool vec, hipStream_t st)
{
    const int unit = dtype == DRF_BF16 ? 8 : 4;
    vec = vec && a.d % unit == 0;
    const int kind = !a.r.columns ? 0 : rope->layout == DRF_ROPE_PAIRS ? 1 : 2;
    a.granule = unit;
    if (kind == 2)
        for (int i = 0; i < rope->n_axes; ++i)
            while (rope->dim[i] / 2 % a.granule) a.granule /= 2;
    return dtype == DRF_BF16 ? launch<bf16_t>(a, norm, kind, vec, st) : launch<float>(a, norm, kind, vec, st);
}

drf_status check_sizes(drf_dtype dtype, int slots, int tokens, int heads, int head_dim)
{
    if (dtype != DRF_F32 && dtype != DRF_BF16) DRF_FAIL(DRF_EINVAL, "unknown dtype");
    if (slots < 0 || tokens < 0 || heads < 1 || head_dim < 1) DRF_FAIL(DRF_EINVAL, "slots and tokens must be >= 0, heads and head_dim >= 1");
    if (head_dim > kMaxD) DRF_FAIL(DRF_ESHAPE, "head_dim must be <= %d (got %d)", kMaxD, head_dim);
    if (heads > 65535) DRF_FAIL(DRF_ESHAPE, "more than 65535 heads");
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
    if ((rc = fill_side("x", x, out, heads, &vec, dtype == DRF_BF16 ? 8 : 4, &a.q)) != DRF_OK) return rc;
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
    if ((rc = fill_side("q", q, q_out, s.q_heads, &vec, unit, &a.q)) != DRF_OK) return rc;
    if ((rc = fill_side("k", k, k_out, s.kv_heads, &vec, unit, &a.k)) != DRF_OK) return rc;
    a.q.scale = cfg->q_scale; a.k.scale = 1.f;
    a.q.gain = cfg->q_gain; a.q.bias = cfg->q_bias; a.k.gain = cfg->k_gain; a.k.bias = cfg->k_bias;
    a.slots = s.slots; a.tokens = s.q_tokens; a.d = s.head_dim; a.lens = s.q_lens; a.eps = (float)cfg->eps;
    return run_heads(a, rope, s.dtype, cfg->norm, vec, (hipStream_t)hip_stream);
}
