// The update of the residual stream between two branches of a block, with the norm behind the one and before the other:
//   z = x_scale x + y_scale gate * after(y),  h = before(z) (1 + scale) + shift
//
// A row's lanes hold it in registers from its load to its stores: mean, then the squares of what is left of it (two sums, so that a large mean costs nothing
// of the variance), each over the lanes without LDS where one wave has a row.  Everything is read and written once: bound by memory.
#include <algorithm>
#include <type_traits>

#include "rows.h"

namespace drf {

namespace {

constexpr int kMaxWidth = 16384;

struct RowNormArgs { int norm; float eps; const float *gain, *bias; };
struct ResidualArgs {
    drf_rows x, y, out, h, gate, shift, scale;
    int rows, tokens, width;
    uint32_t tok_magic; int tok_shift;
    const int32_t* lens;
    float x_scale, y_scale, inv_width;
    RowNormArgs after, before;
};

__device__ inline int div_by(int n, uint32_t magic, int shift) { return magic ? (int)(__umulhi((uint32_t)n, magic) >> shift) : (n >> shift); }

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

template <typename T, int E> struct Piece { typedef T type __attribute__((ext_vector_type(E))); };
template <typename T> struct Piece<T, 1> { typedef T type; };
template <int E, typename T> __device__ inline void load_piece(const T* p, float (&v)[E])
{
    const auto q = *reinterpret_cast<const typename Piece<T, E>::type*>(p);
    if constexpr (E == 1) v[0] = (float)q;
    else
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = (float)q[j];
}
template <int E, typename T> __device__ inline void store_piece(T* p, const float (&v)[E])
{
    typename Piece<T, E>::type q;
    if constexpr (E == 1) q = (T)v[0];
    else
#pragma unroll
        for (int j = 0; j < E; ++j) q[j] = (T)v[j];
    *reinterpret_cast<typename Piece<T, E>::type*>(p) = q;
}

// A lane holds NV pieces of E columns of its row.  MULTI: the workgroup's waves share a row, otherwise each has its own.
template <typename TS, typename TB, int E, int NV, bool MULTI>
__global__ void __launch_bounds__(MULTI ? 512 : 256) residual_norm_kernel(const ResidualArgs a)
{
    __shared__ float part[2][MULTI ? 4 : 1][8];
    const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = MULTI ? threadIdx.x : threadIdx.x & 63, lanes = MULTI ? blockDim.x : 64;
    const int step = MULTI ? gridDim.x : gridDim.x * waves;
    // sum over the row; a row's sums and the next row's have places of their own, so that one barrier is enough for each
    int turn = 0;
    auto total = [&](float v, int at) {
        v = wave_total(v);
        if constexpr (MULTI) {
            if ((threadIdx.x & 63) == 0) part[turn][at][wave] = v;
            __syncthreads();
            v = 0.f;
            for (int w = 0; w < waves; ++w) v += part[turn][at][w];
        }
        return v;
    };
    for (long long row = MULTI ? blockIdx.x : (long long)blockIdx.x * waves + wave; row < a.rows; row += step) {
        const int slot = div_by((int)row, a.tok_magic, a.tok_shift), token = (int)row - slot * a.tokens;
        if (token >= slot_len(a.lens, slot, a.tokens)) continue;    // (the same for all lanes of a row)
        auto at = [&](const drf_rows& t) { return slot * t.slot_stride + token * t.token_stride; };
        turn ^= 1;
        float z[NV][E], y[NV][E];
        auto col = [&](int v) { return (v * lanes + li) * E; };
        auto for_all = [&](auto f) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (col(v) < a.width) f(v, col(v));
        };
        auto load = [&](const auto* p, float (&r)[NV][E]) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (col(v) < a.width) load_piece<E>(p + col(v), r[v]);
                else
#pragma unroll
                    for (int j = 0; j < E; ++j) r[v][j] = 0.f;
            }
        };
        // norm of r in place, without gain and bias
        auto norm = [&](float (&r)[NV][E], const RowNormArgs& n, int first) {
            if (n.norm == DRF_QK_NONE) return;
            float s = 0.f;
            if (n.norm == DRF_QK_LAYER) {
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < E; ++j) s += r[v][j];
                const float mean = total(s, first) * a.inv_width;
                s = 0.f;
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int j = 0; j < E; ++j) r[v][j] = col(v) < a.width ? r[v][j] - mean : 0.f;
            }
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < E; ++j) s = fmaf(r[v][j], r[v][j], s);
            const float inv = 1.f / sqrtf(fmaf(total(s, first + 1), a.inv_width, n.eps));
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < E; ++j) r[v][j] *= inv;
        };
        load((const TS*)a.x.data + at(a.x), z);
        if (a.y.data) {
            load((const TB*)a.y.data + at(a.y), y);
            norm(y, a.after, 0);
            for_all([&](int v, int c) {
                float g[E], t[E];
                if (a.after.gain) {
                    load_piece<E>(a.after.gain + c, t);
#pragma unroll
                    for (int j = 0; j < E; ++j) y[v][j] *= t[j];
                }
                if (a.after.bias) {
                    load_piece<E>(a.after.bias + c, t);
#pragma unroll
                    for (int j = 0; j < E; ++j) y[v][j] += t[j];
                }
                if (a.gate.data) load_piece<E>((const float*)a.gate.data + at(a.gate) + c, g);
                else
#pragma unroll
                    for (int j = 0; j < E; ++j) g[j] = 1.f;
#pragma unroll
                for (int j = 0; j < E; ++j) z[v][j] = fmaf(a.y_scale * g[j], y[v][j], a.x_scale * z[v][j]);
            });
        } else {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < E; ++j) z[v][j] *= a.x_scale;
        }
        if (a.out.data) {
            TS* o = (TS*)a.out.data + at(a.out);
            for_all([&](int v, int c) { store_piece<E>(o + c, z[v]); });
        }
        if (!a.h.data) continue;
        norm(z, a.before, 2);
        TB* o = (TB*)a.h.data + at(a.h);
        for_all([&](int v, int c) {
            float t[E];
            if (a.before.gain) {
                load_piece<E>(a.before.gain + c, t);
#pragma unroll
                for (int j = 0; j < E; ++j) z[v][j] *= t[j];
            }
            if (a.before.bias) {
                load_piece<E>(a.before.bias + c, t);
#pragma unroll
                for (int j = 0; j < E; ++j) z[v][j] += t[j];
            }
            if (a.scale.data) {
                load_piece<E>((const float*)a.scale.data + at(a.scale) + c, t);
#pragma unroll
                for (int j = 0; j < E; ++j) z[v][j] *= 1.f + t[j];
            }
            if (a.shift.data) {
                load_piece<E>((const float*)a.shift.data + at(a.shift) + c, t);
#pragma unroll
                for (int j = 0; j < E; ++j) z[v][j] += t[j];
            }
            store_piece<E>(o + c, z[v]);
        });
    }
}

template <typename TS, typename TB, int E, int NV>
void go(const ResidualArgs& a, int waves, hipStream_t st)
{
    if (waves > 1) {
        const int grid = std::min(a.rows, 1 << 22);
        hipLaunchKernelGGL((residual_norm_kernel<TS, TB, E, NV, true>), dim3(grid), dim3(64 * waves), 0, st, a);
    } else {
        const int per = a.rows >= 4096 ? 4 : 1;                     // few rows go to as many CUs as there are
        const int grid = std::min((a.rows + per - 1) / per, 1 << 22);
        hipLaunchKernelGGL((residual_norm_kernel<TS, TB, E, NV, false>), dim3(grid), dim3(64 * per), 0, st, a);
    }
}

// Up to 32 columns a lane: one wave to 2048, then as many as the width asks for.
template <typename TS, typename TB, int E> void pick(const ResidualArgs& a, hipStream_t st)
{
    const int waves = (a.width + 2047) / 2048, n = (a.width + 64 * waves - 1) / (64 * waves);
    if (n <= 8) go<TS, TB, E, 8 / E>(a, waves, st);
    else if (n <= 24) go<TS, TB, E, 24 / E>(a, waves, st);
    else go<TS, TB, E, 32 / E>(a, waves, st);
}

template <typename TS, typename TB> void pick_piece(const ResidualArgs& a, int e, hipStream_t st)
{
    constexpr int most = sizeof(TS) == 2 ? 8 : 4;
    if (e >= most) pick<TS, TB, most>(a, st);
    else if (e >= 2) pick<TS, TB, 2>(a, st);
    else pick<TS, TB, 1>(a, st);
}

drf_status fill_norm(const char* what, const drf_row_norm& n, RowNormArgs* out)
{
    if (n.norm != DRF_QK_NONE && n.norm != DRF_QK_RMS && n.norm != DRF_QK_LAYER) DRF_FAIL(DRF_EINVAL, "%s: unknown norm", what);
    if (!(n.eps >= 0.0) || !std::isfinite(n.eps)) DRF_FAIL(DRF_EINVAL, "%s: eps must be >= 0", what);
    if (n.norm == DRF_QK_NONE && n.gain) DRF_FAIL(DRF_EINVAL, "%s: a gain without a norm", what);
    if (n.norm != DRF_QK_LAYER && n.bias) DRF_FAIL(DRF_EINVAL, "%s: a bias belongs to DRF_QK_LAYER", what);
    // (an eps that fp32 does not hold is still no zero: a row of zeros stays one)
    *out = { (int)n.norm, n.eps > 0.0 ? std::max((float)n.eps, 1.17549435e-38f) : 0.f, n.gain, n.bias };
    return DRF_OK;
}

// Columns that may be taken at once: the largest of 8, 4, 2, 1 that every address and stride is a multiple of.
void lower_piece(int* e, const drf_rows& t, int size)
{
    if (!t.data) return;
    while (*e > 1 && (reinterpret_cast<uintptr_t>(t.data) % std::min(16, *e * size) || t.slot_stride % *e || t.token_stride % *e)) *e /= 2;
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
    if (!std::isfinite(c.x_scale) || !std::isfinite(c.y_scale)) DRF_FAIL(DRF_EINVAL, "x_scale and y_scale must be finite");
    ResidualArgs a{};
    if ((rc = fill_norm("after", c.after, &a.after)) != DRF_OK || (rc = fill_norm("before", c.before, &a.before)) != DRF_OK) return rc;
    if (c.slots == 0 || c.tokens == 0) return DRF_OK;
    auto take = [&](const drf_rows* t) { return t ? used_rows(*t, c.slots, c.tokens) : drf_rows{}; };
    a.x = take(x); a.y = take(y); a.out = take(out); a.h = take(h);
    a.gate = take(&c.gate); a.shift = take(&c.shift); a.scale = take(&c.scale);
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
    int e = 8;
    while (c.width % e) e /= 2;
    const int ss = c.stream == DRF_BF16 ? 2 : 4, bs = c.branch == DRF_BF16 ? 2 : 4;
    lower_piece(&e, a.x, ss); lower_piece(&e, a.out, ss); lower_piece(&e, a.y, bs); lower_piece(&e, a.h, bs);
    for (const drf_rows& t : { a.gate, a.shift, a.scale, drf_rows{ (void*)a.after.gain, 0, 0 }, drf_rows{ (void*)a.after.bias, 0, 0 },
                               drf_rows{ (void*)a.before.gain, 0, 0 }, drf_rows{ (void*)a.before.bias, 0, 0 } })
        lower_piece(&e, t, 4);
    hipStream_t st = (hipStream_t)hip_stream;
    if (c.stream == DRF_BF16) pick_piece<bf16_t, bf16_t>(a, e, st);
    else if (c.branch == DRF_BF16) pick_piece<float, bf16_t>(a, e, st);
    else pick_piece<float, float>(a, e, st);
    DRF_HIP(hipGetLastError());
    return DRF_OK;
}
