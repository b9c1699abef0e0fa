// The update of the residual stream between two branches of a block, with the norm behind the one and before the other:
//   z = x_scale x + y_scale gate * after(y),  h = before(z) (1 + scale) + shift
//
// A row's lanes hold it in registers from its load to its stores: mean, then the squares of what is left of it (two sums, so that a large mean costs nothing
// of the variance), each over the lanes without LDS where one wave has a row.  Everything is read and written once: bound by memory.  6 x 4096 x 1152, stream in fp32, branch in
// bf16, LayerNorm before (340 MB): 64.6 us, 5.26 TB/s;  4 x 16384 x 1536 in bf16, RMS on both sides (805 MB): 143 us, 5.6;  a large copy: 5.18.  One row: 4.4 us, a launch.
// Modulation by token in fp32 doubles the bytes of the first of these: 679 MB, 130 us, 5.2 TB/s.  Rows on a workgroup each: 4 x 4096 of 2560 in bf16, RMS twice (336 MB) 85 us, 3.9;
// of 4096 as the first of these (805 MB) 158, 5.1; 2 x 2048 of 8192 in fp32, LayerNorm twice (537 MB) 129, 4.2.
#include <algorithm>
#include <type_traits>

#include "gemm_device.h"
#include "rows.h"

namespace drf {

namespace {

constexpr int kMaxWidth = 16384;

// A row's squares and their sum are taken in fp32 as they are where that holds them: the sum is finite, and either above kFewSquares (what its smallest terms lose to
// underflow, 16384 of 2^-126 at most, is 2^-29 of it) or of no account beside an eps of kMuchEps or more.  Other rows have a power of two taken out of them first.
constexpr float kFewSquares = 1e-25f, kMuchEps = 1e-30f;
constexpr float kLeastEps = 1.17549435e-38f;        // (an eps that fp32 does not hold is still no zero: a row of zeros stays one)
struct RowNormArgs { int norm; float eps, eps_part; int eps_exp; const float *gain, *bias; };     // eps_part 2^eps_exp: eps as it was given
struct ResidualArgs {
    drf_rows x, y, out, h, gate, shift, scale;
    int rows, tokens, width;
    int first, slot_tiles;              // workgroup that a launch begins with; workgroups a slot
    uint32_t tok_magic; int tok_shift;
    const int32_t* lens;
    float x_scale, y_scale, inv_width;
    RowNormArgs after, before;
};

// Sum over a wave's lanes, in all of them: quads, halves of 16, 16, and the rows of 16 by swaps.  No LDS, some 6 dependent adds.
__device__ inline float wave_total(float v)
{
    auto dpp = [](float x, auto ctrl) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true)); };
    v += dpp(v, std::integral_constant<int, 0xb1>{});               // quad_perm 1 0 3 2
    v += dpp(v, std::integral_constant<int, 0x4e>{});               // quad_perm 2 3 0 1
    v += dpp(v, std::integral_constant<int, 0x141>{});              // mirror of 8
    v += dpp(v, std::integral_constant<int, 0x140>{});              // mirror of 16
    const int b16 = __builtin_bit_cast(int, v);
    const auto r = __builtin_amdgcn_permlane16_swap(b16, b16, false, false);
    v = __builtin_bit_cast(float, (int)r[0]) + __builtin_bit_cast(float, (int)r[1]);
    const int b32 = __builtin_bit_cast(int, v);
    const auto s = __builtin_amdgcn_permlane32_swap(b32, b32, false, false);
    return __builtin_bit_cast(float, (int)s[0]) + __builtin_bit_cast(float, (int)s[1]);
}

__device__ inline float wave_most(float v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

// E columns of a row at any address that is a multiple of an element: the memory system takes 16 bytes at once from there too.
template <typename T, int E> struct Piece { typedef T type __attribute__((ext_vector_type(E), aligned(sizeof(T)))); };
template <typename T> struct Piece<T, 1> { typedef T type __attribute__((ext_vector_type(1))); };
template <int E, typename T> __device__ inline typename Piece<T, E>::type load_piece(const T* p) { return *reinterpret_cast<const typename Piece<T, E>::type*>(p); }
template <int E, typename T> __device__ inline void store_piece(T* p, const float (&v)[E])
{
    typename Piece<T, E>::type q;
#pragma unroll
    for (int j = 0; j < E; ++j) q[j] = (T)v[j];
    *reinterpret_cast<typename Piece<T, E>::type*>(p) = q;
}

// A lane holds NV pieces of E columns of its row; the piece that a row ends inside of begins E columns before that end, and its columns that are its
// neighbour's too count in the neighbour's sums alone.  What a slot's rows have in common comes together in four numbers a column:
//   z = x_scale x + g n(y) + gb,  h = s n(z) + sb:   g = y_scale gate gain, gb = y_scale gate bias (BIAS),  s = gain (1 + scale), sb = bias (1 + scale) + shift
// FORM: ROW_WAVE a wave a row, ROW_GROUP the workgroup's waves share a row, ROW_STAGED a wave a row of the same slot for all waves of the workgroup, which form
// those numbers once, in LDS, while their rows are on the way: from the near cache for every row they are twice what the rows themselves read
// (6 x 4096 x 1152, stream in fp32, branch in bf16, 340 MB, LayerNorm before: 110 us, without modulation 68).
enum { ROW_WAVE = 0, ROW_GROUP = 1, ROW_STAGED = 2 };
template <typename TS, typename TB, int E, int NV, int FORM, bool BIAS>
__global__ void __launch_bounds__(512) residual_norm_kernel(const ResidualArgs a)
{
    constexpr bool GROUP = FORM == ROW_GROUP, STAGED = FORM == ROW_STAGED;
    constexpr int KINDS = BIAS ? 4 : 3, ROW = NV * 64 * E;
    __shared__ float part[GROUP ? 8 : 1][8];
    __shared__ __attribute__((aligned(32))) float table[STAGED ? KINDS * ROW : 1];
    const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = GROUP ? threadIdx.x : threadIdx.x & 63, lanes = GROUP ? blockDim.x : 64;
    int slot, token;
    if constexpr (STAGED) {
        const int id = a.first + blockIdx.x;
        slot = id / a.slot_tiles;
        token = (id - slot * a.slot_tiles) * waves + wave;
    } else {
        const int row = GROUP ? a.first + blockIdx.x : (a.first + blockIdx.x) * waves + wave;
        slot = fast_div(row, a.tok_magic, a.tok_shift);
        token = row - slot * a.tokens;
        if (row >= a.rows) return;
    }
    const bool live = token < slot_len(a.lens, slot, a.tokens);    // (the same for all lanes of a row)
    if (!STAGED && !live) return;
    auto total = [&](float v, int at) {
        v = wave_total(v);
        if constexpr (GROUP) {
            if ((threadIdx.x & 63) == 0) part[at][wave] = v;
            __syncthreads();
            v = 0.f;
            for (int w = 0; w < waves; ++w) v += part[at][w];
        }
        return v;
    };
    int skip[NV], col[NV];                          // a piece's columns that are its neighbour's (E: it is not there), its first column
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * lanes + li) * E, left = a.width - c;
        skip[v] = left >= E ? 0 : left > 0 ? E - left : E;
        col[v] = left >= E ? c : a.width - E;
    }
    auto squares = [&](const float (&r)[NV][E]) {
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float t = j >= skip[v] ? r[v][j] : 0.f;
                s = fmaf(t, t, s);
            }
        return s;
    };
    auto norm = [&](float (&r)[NV][E], const RowNormArgs& n, int first) {
        if (n.norm == DRF_QK_NONE) return;
        if (n.norm == DRF_QK_LAYER) {
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < E; ++j) s += j >= skip[v] ? r[v][j] : 0.f;
            const float mean = total(s, first) * a.inv_width;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < E; ++j) r[v][j] -= mean;
        }
        float s = total(squares(r), first + 1), eps = n.eps;
        if (__builtin_expect(!(s < INFINITY) || (s < kFewSquares && eps < kMuchEps), 0)) {     // (the same for all lanes of the row)
            float most = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < E; ++j) most = fmaxf(most, j >= skip[v] ? fabsf(r[v][j]) : 0.f);
            most = wave_most(most);
            if constexpr (GROUP) {
                if ((threadIdx.x & 63) == 0) part[first + 2][wave] = most;
                __syncthreads();
                for (int w = 0; w < waves; ++w) most = fmaxf(most, part[first + 2][w]);
            }
            if (most < INFINITY) {                  // (a row with an infinity: no number there, zeros beside it)
                // x / sqrt(mean x^2 + eps) with x = 2^e t, |t| < 4: t / sqrt(mean t^2 + eps 2^-2e).  The lowest e that any fp32 row needs keeps an eps below kMuchEps finite
                const int e = max(-110, min(126, (int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127));
                const float f = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < E; ++j) r[v][j] *= f;
                s = total(squares(r), first + 3);
                eps = n.eps > 0.f ? fmaxf(ldexpf(n.eps_part, n.eps_exp - 2 * e), kLeastEps) : 0.f;
            }
        }
        const float inv = 1.f / sqrtf(fmaf(s, a.inv_width, eps));
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < E; ++j) r[v][j] *= inv;
    };
    const bool has_y = a.y.data != nullptr, has_h = a.h.data != nullptr;
    typename Piece<TS, E>::type px[NV];
    typename Piece<TB, E>::type py[NV];
    if (live) {
        const TS* x = (const TS*)a.x.data + slot * a.x.slot_stride + token * a.x.token_stride;
        const TB* y = (const TB*)a.y.data + slot * a.y.slot_stride + token * a.y.token_stride;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (skip[v] < E) px[v] = load_piece<E>(x + col[v]);
            if (has_y && skip[v] < E) py[v] = load_piece<E>(y + col[v]);
        }
    }
    // a parameter's columns, or what stands for one that is not there
    auto column = [&](const float* p, int v, float none, float (&out)[E]) {
#pragma unroll
        for (int j = 0; j < E; ++j) out[j] = none;
        if (p && skip[v] < E) {
            const auto q = load_piece<E>(p + col[v]);
#pragma unroll
            for (int j = 0; j < E; ++j) out[j] = q[j];
        }
    };
    auto row_of = [&](const drf_rows& t) { return t.data ? (const float*)t.data + slot * t.slot_stride + token * t.token_stride : nullptr; };
    const float *gate = row_of(a.gate), *scale = row_of(a.scale), *shift = row_of(a.shift);
    auto branch = [&](int v, float (&g)[E], float (&gb)[E]) {
        float t[E], u[E];
        column(gate, v, 1.f, g);
        column(a.after.gain, v, 1.f, t);
        if constexpr (BIAS) column(a.after.bias, v, 0.f, u);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            g[j] *= a.y_scale;
            if constexpr (BIAS) gb[j] = g[j] * u[j];
            g[j] *= t[j];
        }
    };
    auto next_in = [&](int v, float (&s)[E], float (&sb)[E]) {
        float t[E], u[E];
        column(scale, v, 0.f, s);
        column(shift, v, 0.f, sb);
        column(a.before.gain, v, 1.f, t);
        column(a.before.bias, v, 0.f, u);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            s[j] += 1.f;
            sb[j] = fmaf(u[j], s[j], sb[j]);
            s[j] *= t[j];
        }
    };
    auto keep = [&](int kind, int v, const float (&r)[E]) { store_piece<E>(table + kind * ROW + (v * 64 + li) * E, r); };
    auto kept = [&](int kind, int v, float (&r)[E]) {
        const auto q = load_piece<E>(table + kind * ROW + (v * 64 + li) * E);
#pragma unroll
        for (int j = 0; j < E; ++j) r[j] = q[j];
    };
    if constexpr (STAGED) {
        // piece v of both sides by waves of their own, as far as there are
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float p[E], q[E];
            if (has_y && (2 * v) % waves == wave) {
                branch(v, p, q);
                keep(0, v, p);
                if constexpr (BIAS) keep(3, v, q);
            }
            if (has_h && (2 * v + 1) % waves == wave) {
                next_in(v, p, q);
                keep(1, v, p);
                keep(2, v, q);
            }
        }
        __syncthreads();
        if (!live) return;
    }
    float z[NV][E], y[NV][E];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < E; ++j) {
            z[v][j] = skip[v] < E ? (float)px[v][j] * a.x_scale : 0.f;
            y[v][j] = has_y && skip[v] < E ? (float)py[v][j] : 0.f;
        }
    if constexpr (GROUP) __syncthreads();           // (a row in its own place: all of it is read before any of it is written)
    if (has_y) {
        norm(y, a.after, 0);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float g[E], gb[E];
            if constexpr (STAGED) {
                kept(0, v, g);
                if constexpr (BIAS) kept(3, v, gb);
            } else branch(v, g, gb);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if constexpr (BIAS) z[v][j] += gb[j];
                z[v][j] = fmaf(g[j], y[v][j], z[v][j]);
            }
        }
        if (a.out.data) {
            TS* o = (TS*)a.out.data + slot * a.out.slot_stride + token * a.out.token_stride;
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (skip[v] < E) store_piece<E>(o + col[v], z[v]);
        }
    }
    if (!has_h) return;
    norm(z, a.before, 4);
    TB* o = (TB*)a.h.data + slot * a.h.slot_stride + token * a.h.token_stride;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        float s[E], sb[E];
        if constexpr (STAGED) { kept(1, v, s); kept(2, v, sb); }
        else next_in(v, s, sb);
#pragma unroll
        for (int j = 0; j < E; ++j) z[v][j] = fmaf(z[v][j], s[j], sb[j]);
        if (skip[v] < E) store_piece<E>(o + col[v], z[v]);
    }
}

template <typename TS, typename TB, int E, int NV, int FORM>
void go(ResidualArgs& a, int waves, hipStream_t st)
{
    a.slot_tiles = (a.tokens + waves - 1) / waves;
    const int all = FORM == ROW_STAGED ? a.rows / a.tokens * a.slot_tiles : FORM == ROW_GROUP ? a.rows : (a.rows + waves - 1) / waves;
    const int most = 1 << 22;                                       // (a launch holds fewer than 2^32 threads)
    for (a.first = 0; a.first < all; a.first += most) {
        const int grid = std::min(all - a.first, most);
        if (a.after.bias) hipLaunchKernelGGL((residual_norm_kernel<TS, TB, E, NV, FORM, true>), dim3(grid), dim3(64 * waves), 0, st, a);
        else hipLaunchKernelGGL((residual_norm_kernel<TS, TB, E, NV, FORM, false>), dim3(grid), dim3(64 * waves), 0, st, a);
    }
}

template <typename TS, typename TB, int E, int NV> void go_rows(ResidualArgs& a, hipStream_t st)
{
    // fewer rows than the chip holds waves: a row each, its numbers for itself
    constexpr int W = 8, T = 2048;
    const bool each = (a.gate.data && a.gate.token_stride) || (a.scale.data && a.scale.token_stride) || (a.shift.data && a.shift.token_stride);
    if (!each && a.rows >= T && a.tokens >= W) go<TS, TB, E, NV, ROW_STAGED>(a, W, st);
    else go<TS, TB, E, NV, ROW_WAVE>(a, a.rows < 2048 ? 1 : 4, st);
}

// Up to 32 columns a lane: one wave to 2048, then as many as the width asks for.
template <typename TS, typename TB> void pick(ResidualArgs& a, hipStream_t st)
{
    constexpr int E = sizeof(TS) == 2 ? 8 : 4;
    if (a.width < E) return go<TS, TB, 1, 1, ROW_WAVE>(a, 4, st);
    const int waves = (a.width + 2047) / 2048, n = (a.width + 64 * E * waves - 1) / (64 * E * waves);
    if (waves > 1) {
        if (n * E <= 24) go<TS, TB, E, 24 / E, ROW_GROUP>(a, waves, st);
        else go<TS, TB, E, 32 / E, ROW_GROUP>(a, waves, st);
    } else if (n * E <= 8) go_rows<TS, TB, E, 8 / E>(a, st);
    else if (n * E <= 16) go_rows<TS, TB, E, 16 / E>(a, st);
    else if (E == 4 && n <= 5) go_rows<TS, TB, E, E == 4 ? 5 : 3>(a, st);
    else if (n * E <= 24) go_rows<TS, TB, E, 24 / E>(a, st);
    else go_rows<TS, TB, E, 32 / E>(a, st);
}

drf_status fill_norm(const char* what, const drf_row_norm& n, RowNormArgs* out)
{
    if (n.norm != DRF_QK_NONE && n.norm != DRF_QK_RMS && n.norm != DRF_QK_LAYER) DRF_FAIL(DRF_EINVAL, "%s: unknown norm", what);
    if (!(n.eps >= 0.0) || !std::isfinite(n.eps)) DRF_FAIL(DRF_EINVAL, "%s: eps must be >= 0", what);
    if (n.norm == DRF_QK_NONE && n.gain) DRF_FAIL(DRF_EINVAL, "%s: a gain without a norm", what);
    if (n.norm != DRF_QK_LAYER && n.bias) DRF_FAIL(DRF_EINVAL, "%s: a bias belongs to DRF_QK_LAYER", what);
    int exp = 0;
    const float part = (float)std::frexp(n.eps, &exp);
    *out = { (int)n.norm, n.eps > 0.0 ? std::max((float)n.eps, kLeastEps) : 0.f, part, exp, n.gain, n.bias };
    return DRF_OK;
}

}  // namespace

}  // namespace drf

using namespace drf;

extern "C" drf_status drf_residual_norm(const drf_residual_config* cfg, const drf_rows* x, const drf_rows* y, const drf_rows* out, const drf_rows* h,
                                        void* hip_stream)
{
    if (!cfg) DRF_FAIL(DRF_EINVAL, "NULL configuration");
    const drf_residual_config& c = *cfg;
    if (!known_dtype(c.stream) || !known_dtype(c.branch)) DRF_FAIL(DRF_EINVAL, "unknown dtype");
    if (c.stream == DRF_BF16 && c.branch == DRF_F32) DRF_FAIL(DRF_EUNSUPPORTED, "a bf16 stream with an fp32 branch");
    drf_status rc = check_rows_sizes(c.slots, c.tokens);
    if (rc != DRF_OK) return rc;
    if (c.width < 1) DRF_FAIL(DRF_EINVAL, "width must be >= 1");
    if (c.width > kMaxWidth) DRF_FAIL(DRF_ESHAPE, "width must be <= %d (got %d)", kMaxWidth, c.width);
    if (!std::isfinite(c.x_scale) || (y && !std::isfinite(c.y_scale))) DRF_FAIL(DRF_EINVAL, "x_scale and y_scale must be finite");
    ResidualArgs a{};
    if (y && (rc = fill_norm("after", c.after, &a.after)) != DRF_OK) return rc;
    if ((rc = fill_norm("before", c.before, &a.before)) != DRF_OK) return rc;
    if (c.slots == 0 || c.tokens == 0) return DRF_OK;
    auto take = [&](const drf_rows* t) { return t ? used_rows(*t, c.slots, c.tokens) : drf_rows{}; };
    a.x = take(x); a.y = take(y); a.out = take(out); a.h = take(h);
    a.gate = take(y ? &c.gate : nullptr); a.shift = take(&c.shift); a.scale = take(&c.scale);
    if (!a.x.data || (y && !y->data) || (out && !out->data) || (h && !h->data)) DRF_FAIL(DRF_EINVAL, "NULL tensor");
    if (!a.out.data && !a.h.data) DRF_FAIL(DRF_EINVAL, "neither the stream nor its norm is asked for");
    if (!a.y.data && a.out.data) DRF_FAIL(DRF_EINVAL, "a stream is stored where a branch is added to it");
    auto alike = [](const drf_rows& p, const drf_rows& q) { return p.data != q.data || (p.slot_stride == q.slot_stride && p.token_stride == q.token_stride); };
    for (const drf_rows* o : { &a.out, &a.h })
        if (o->data && rows_overlap(*o, c.slots, c.tokens, c.width)) DRF_FAIL(DRF_EINVAL, "rows of an output lie on one another");
    if ((a.out.data && !alike(a.out, a.x)) || (a.h.data && a.y.data && !alike(a.h, a.y)))
        DRF_FAIL(DRF_EINVAL, "input and output share an address but not their strides");
    if (a.out.data == a.h.data || (a.out.data && a.out.data == a.y.data) || a.h.data == a.x.data) DRF_FAIL(DRF_EINVAL, "an output lies on another tensor");
    a.rows = c.slots * c.tokens; a.tokens = c.tokens; a.width = c.width;
    make_fast_div(c.tokens, &a.tok_magic, &a.tok_shift);
    a.lens = c.lens;
    a.x_scale = c.x_scale; a.y_scale = c.y_scale; a.inv_width = 1.f / (float)c.width;
    hipStream_t st = (hipStream_t)hip_stream;
    if (c.stream == DRF_BF16) pick<bf16_t, bf16_t>(a, st);
    else if (c.branch == DRF_BF16) pick<float, bf16_t>(a, st);
    else pick<float, float>(a, st);
    DRF_HIP(hipGetLastError());
    return DRF_OK;
}
