// bf16 products of rows [slots][tokens][K] with weights, for the feed-forward block and the projections with adapters: BM x BN tiles, operands by direct
// copies to LDS NS - 1 steps of 64 of the inner axis ahead, 16x16x32 matrix instructions, waves as WM x WN.
//
// The loop is that of the framework's other products: the matrix instructions of a step in groups of one weight fragment, whose LDS read is issued
// R - 1 groups ahead, one barrier a step that far before its end, one copy instruction a group.  What is this kernel's own:
//  - rows by slot and token with strides: a lane's copies have 32-bit offsets from its workgroup's first slot (or first row, where tiles keep to a slot);
//  - an inner axis that is a multiple of 8 only: the last step's copies repeat the row's last 16 bytes, and zeros are written over them once they have
//    landed (in both operands: nothing times an infinity that lies beside);
//  - LIN_GLU: rows of a weight tile are 16 of the gate, 16 of the value, and so on, so that a lane ends with both of a column; half the columns go out;
//  - LIN_ADAPT: where a tile keeps to a slot its adapter is more steps of the loop, 32 columns of the rank each: 64 columns of a row are the upper and
//    the lower halves of its x A^T, those of a weight row twice the same of B.  Elsewhere the adapters are added to the finished sums (add_adapters);
//  - the result goes out in whole rows through the idle stages, rows that are not there left out.
// Large products are bound by the clock under the matrix unit (gate and value of 65536 rows, 1152 x 9216, on 256 x 256: 1190 to 1300 us, 1.07 to 1.17 PFLOP/s with the activation), single
// rounds by first copies and store (12 x 256 rows, 384 x 2 x 1536: 18 us on 144 tiles, of which the matrix unit is busy for 3).  Smaller ones are for the rounds
// that they fill better: 19 x 77 rows, 1024 x 2304 with adapters of rank 24, 18 us on 216 tiles of 128 x 128.
#pragma once
#include "linear_direct.h"
#include "linear_wide.h"

namespace drf {

namespace {

template <int BM, int BN, int NS, int WM, int WN, int KIND>
__global__ void __launch_bounds__(WM * WN * 64) linear_tile_kernel(const LinArgs a)
{
    constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, MI = TM / 16, NI = TN / 16;
    constexpr int STAGE = (BM + BN) * 128, SEG = (BM + BN) / 8, LPT = SEG / NW, GROUP_M = 8;
    constexpr int ON = KIND == LIN_GLU ? TN / 2 : TN, PITCH = ON * 2 + 16, CH = ON / 8;        // columns of a wave's result; its rows in LDS, in 16-byte pieces
    constexpr int PASS = NW * TM * PITCH <= NS * STAGE ? TM : 32;     // rows of it at a time
    static_assert(BN % 64 == 0 && SEG % NW == 0 && LPT % 2 == 0 && BM <= NW * 64 && NW * PASS * PITCH <= NS * STAGE, "tile shape");
    extern __shared__ __attribute__((aligned(128))) unsigned char smem[];   // stages | bias of the tile's weight rows | where its rows go
    float* bias = reinterpret_cast<float*>(smem + NS * STAGE);
    uint32_t* out_at = reinterpret_cast<uint32_t*>(bias + BN);

    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave % WM, wn = wave / WM;
    int tm, tn;
    {
        // tiles in groups of GROUP_M rows of them, consecutive ones on one XCD
        const int nb = gridDim.x;
        const long long idx = a.first + item_by_xcd(blockIdx.x, nb);
        const long long per_group = (long long)GROUP_M * a.tiles_n, group = idx / per_group;
        const int in = (int)(idx - group * per_group), first_m = (int)group * GROUP_M;
        const int gsz = a.tiles_m - first_m < GROUP_M ? a.tiles_m - first_m : GROUP_M;
        tm = first_m + in % gsz;
        tn = in / gsz;
    }
    const int group = tm / a.slot_tiles, row0 = (tm - group * a.slot_tiles) * BM, n0 = tn * (KIND == LIN_GLU ? BN / 2 : BN);
    const int nk = (a.K + 63) / 64, chunks = (a.K & 63) / 8;        // pieces of the last step; 0: all eight
    const int ad = KIND == LIN_ADAPT && a.in_loop ? __builtin_amdgcn_readfirstlane(adapter_of(a, group)) : -1;
    const int nt = nk + (ad >= 0 ? a.low_cols / 32 : 0), bound = KIND == LIN_ADAPT ? nt : nk;   // steps of the product and of the adapter
    int slot0, token0;
    const bool some = locate_row(a, group, row0, slot0, token0);
    if (a.slot_rows == a.tokens) {
        if (!some) return;                                          // the slot ends before this tile
    } else token0 = 0;
    const char* x0 = (const char*)a.x.data + (slot0 * a.x.slot_stride + token0 * a.x.token_stride) * 2;
    char* out0 = (char*)a.out.data + (slot0 * a.out.slot_stride + token0 * a.out.token_stride) * 2;

    // A wave's copies: LPT instructions of 8 rows; chunk c of row r sits at position c ^ ((r / 2) % 8).
    const int prow = lane >> 3, ppos = lane & 7;
    uint32_t voff[LPT], over[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int chunk = ppos ^ ((p * 4 + prow / 2) & 7);
        over[p] = chunks && chunk >= chunks ? (uint32_t)(chunk - chunks + 1) * 16u : 0u;
    }
#pragma unroll
    for (int i = 0; i < LPT; ++i) {
        const int r = (wave * LPT + i) * 8 + prow, chunk = ppos ^ ((r / 2) & 7);
        if ((wave * LPT + i) * 8 < BM) {
            int slot, token;
            if (!locate_row(a, group, row0 + r, slot, token)) { slot = slot0; token = token0; }
            voff[i] = (uint32_t)(((slot - slot0) * a.x.slot_stride + (token - token0) * a.x.token_stride) * 2) + (uint32_t)chunk * 16u;
        } else {
            int n = r - BM;
            if constexpr (KIND == LIN_GLU) n = n / 32 * 16 + n % 16;
            n = n0 + n < a.N ? n : a.N - 1 - n0;
            voff[i] = (uint32_t)n * (uint32_t)a.K * 2u + (uint32_t)chunk * 16u;
        }
    }
    const char* w0 = (const char*)a.w + (size_t)n0 * a.K * 2;
    const ptrdiff_t to_x = (ptrdiff_t)((uintptr_t)x0 - (uintptr_t)w0), to_value = (ptrdiff_t)a.N * a.K * 2;
    const char* low0 = (const char*)a.low + ((size_t)slot0 * a.tokens + row0) * a.low_cols * 4;
    const char* b0 = (const char*)a.b + ((size_t)(ad < 0 ? 0 : ad) * a.N + n0) * a.rank * 2;
    const ptrdiff_t to_low = (ptrdiff_t)((uintptr_t)low0 - (uintptr_t)b0);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(DRF_LDS_AS unsigned char*)smem;
    // PLAIN: a step of the product whose rows do not end in it
    auto issue_one = [&](auto ic, auto plain_c, int kt, int stage) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value;
        constexpr bool PLAIN = decltype(plain_c)::value;
        const int g = wave * LPT + i;
        // (sums: a choice between the three addresses would keep them, and everything beside them, in memory)
        const bool of_x = g * 8 < BM, second = KIND == LIN_GLU && !of_x && ((g - BM / 8) & 2);
        const char* base = w0 + (of_x ? to_x : 0) + (second ? to_value : 0) + (size_t)kt * 128;
        uint32_t vo = voff[i];
        if constexpr (!PLAIN) {
            if (KIND == LIN_ADAPT && kt >= nk) {
                const int r = g * 8 + prow, chunk = ppos ^ ((r / 2) & 7), e = kt - nk, left = (a.rank - 32 * e) / 8;
                base = b0 + (of_x ? to_low : 0) + e * 64;
                if (of_x) vo = (uint32_t)((row0 + r < a.tokens ? r : 0) * a.low_cols * 4 + (chunk & 3) * 16 + (chunk & 4 ? a.low_cols * 2 : 0));
                else vo = (uint32_t)((n0 + r - BM < a.N ? r - BM : a.N - 1 - n0) * a.rank * 2 + ((chunk & 3) < left ? chunk & 3 : left - 1) * 16);
            } else if (chunks && kt == nk - 1) vo -= over[i & 1];
        }
        const uint32_t dst = lds0 + (uint32_t)(stage * STAGE + g * 1024);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(dst), "v"(vo), "s"(base) : "memory");
    };
    auto issue = [&](auto plain_c, int kt, int stage) __attribute__((always_inline)) {
        static_for<0, LPT>([&](auto ic) __attribute__((always_inline)) { issue_one(ic, plain_c, kt, stage); });
    };
    constexpr std::true_type YES{};
    constexpr std::false_type NO{};
    // step kt has landed for every wave: zeros behind the end of its rows, if they end in it
    auto cut = [&](int kt, int stage) __attribute__((always_inline)) {
        const bool low = KIND == LIN_ADAPT && kt >= nk;
        const int from = low ? (a.rank - 32 * (kt - nk)) / 8 : chunks;
        if (low ? from >= 4 : !chunks || kt != nk - 1) return;
        for (int r = tid + (low ? BM : 0); r < BM + BN; r += NW * 64)
            for (int c = from; c < (low ? 4 : 8); ++c) {
                *reinterpret_cast<u32x4*>(smem + stage * STAGE + r * 128 + (c ^ ((r / 2) & 7)) * 16) = (u32x4){ 0, 0, 0, 0 };
                if (low) *reinterpret_cast<u32x4*>(smem + stage * STAGE + r * 128 + ((c + 4) ^ ((r / 2) & 7)) * 16) = (u32x4){ 0, 0, 0, 0 };
            }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };

    f32x4 acc[NI][MI];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < MI; ++j) acc[i][j] = (f32x4){ 0.f, 0.f, 0.f, 0.f };

    constexpr int G = 2 * NI;
    constexpr int R = G % 6 == 0 && NI >= 6 ? 6 : G % 4 == 0 && NI >= 4 ? 4 : 2, D = R - 1;
    static_assert(G % R == 0 && D < NI && D + MI <= 15, "ring size");
    constexpr int HEAD0 = D < LPT ? D : LPT;
    constexpr bool kSpread = NS == 2 && LPT - HEAD0 <= G - D;
    constexpr int HEAD = kSpread ? HEAD0 : LPT, TAIL = LPT - HEAD;
    u32x4 fa[2][MI], fw[R];
    uint32_t a_addr[2], w_addr[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        const uint32_t pos = (uint32_t)(l16 * 128 + (((ks * 4 + quarter) ^ ((l16 / 2) & 7)) * 16));
        a_addr[ks] = lds0 + (uint32_t)(wm * TM * 128) + pos;
        w_addr[ks] = lds0 + (uint32_t)((BM + wn * TN) * 128) + pos;
    }
    auto fetch = [&](auto pc, const uint32_t (&aa)[2], const uint32_t (&wa)[2]) __attribute__((always_inline)) {
        constexpr int p = decltype(pc)::value, ks = p / NI, i = p % NI;
        if constexpr (i == 0)
            static_for<0, MI>([&](auto jc) __attribute__((always_inline)) {
                constexpr int j = decltype(jc)::value;
                lds_read16<j * 2048>(fa[ks & 1][j], aa[ks]);
            });
        lds_read16<i * 2048>(fw[p % R], wa[ks]);
    };

    stage_bias<BN, NW, KIND>(a, bias, n0, wave);
#pragma unroll
    for (int t = 0; t < NS - 1; ++t)
        if (t < bound) issue(NO, t, t);
    if (tid < BM) {
        int slot, token;
        const bool live = locate_row(a, group, row0 + tid, slot, token);
        out_at[tid] = live ? (uint32_t)(((slot - slot0) * a.out.slot_stride + (token - token0) * a.out.token_stride) * 2) : 0xffffffffu;
    }
    if (NS > 2 && bound >= NS - 1) wait_vmcnt<LPT * (NS - 2)>(); else wait_vmcnt<0>();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    cut(0, 0);
    static_for<0, NI * MI>([&](auto pc) __attribute__((always_inline)) { constexpr int p = decltype(pc)::value; hold_acc<false>(acc[p / MI][p % MI]); });
    settle_mfma();
    if (NS - 1 < bound) issue(NO, NS - 1, NS - 1);
    static_for<0, D>([&](auto pc) { fetch(pc, a_addr, w_addr); });
    int cs = 0;                                     // stage of step kt
    // One step.  PLAIN: the copies that it starts are of plain steps, and there are some.  (Where a lane's offset is made anew for a copy, the copy has to have read it before
    // the register can take a fragment: 0.2 us a step, so the other steps are a loop of their own.)
    auto step = [&](auto plain_c, int kt) __attribute__((always_inline)) {
        constexpr bool PLAIN = decltype(plain_c)::value;
        const int ns = cs + 1 == NS ? 0 : cs + 1;
        const uint32_t co = (uint32_t)cs * (uint32_t)STAGE, no = (uint32_t)ns * (uint32_t)STAGE;
        uint32_t ca[2], cw[2], na[2], nw[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) { ca[ks] = a_addr[ks] + co; cw[ks] = w_addr[ks] + co; na[ks] = a_addr[ks] + no; nw[ks] = w_addr[ks] + no; }
        static_for<0, G>([&](auto gc) __attribute__((always_inline)) {
            constexpr int g = decltype(gc)::value;
            if constexpr (g + D == G) {
                // step kt + 1 has landed and this wave's reads of step kt are complete, for every wave after the barrier: kt's stage may be filled again
                if (NS > 2 && (PLAIN || kt + NS - 1 < bound)) wait_vmcnt<LPT * (NS - 2)>(); else wait_vmcnt<0>();
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                if constexpr (!PLAIN) {
                    if (kt + 1 < bound) cut(kt + 1, ns);
                }
                if constexpr (!kSpread) {
                    if (PLAIN || kt + NS < bound) issue(plain_c, kt + NS, cs);
                }
            }
            if constexpr (kSpread) {
                if constexpr (g >= G - D && g - (G - D) < HEAD) {
                    if (PLAIN || kt + NS < bound) issue_one(std::integral_constant<int, g - (G - D)>{}, plain_c, kt + NS, cs);
                } else if constexpr (g < G - D && g < TAIL) {
                    if (kt >= 1 && (PLAIN || kt + 1 < bound)) issue_one(std::integral_constant<int, HEAD + g>{}, plain_c, kt + 1, ns);
                }
            }
            // (in the last step the positions beyond it read the idle stage: LDS that is there, values unused)
            if constexpr (g + D < G) fetch(std::integral_constant<int, g + D>{}, ca, cw);
            else fetch(std::integral_constant<int, g + D - G>{}, na, nw);
            __builtin_amdgcn_sched_barrier(0);
            constexpr int later = D + (((g + D) / NI) != (g / NI) ? MI : 0);     // reads issued behind this group's
            if constexpr (g % NI == 0) wait_frags<later, MI>(fw[g % R], fa[(g / NI) & 1]);
            else wait_frag<later>(fw[g % R]);
            static_for<0, MI>([&](auto jc) __attribute__((always_inline)) {
                constexpr int j = (g & 1) ? MI - 1 - decltype(jc)::value : decltype(jc)::value;
                mfma<false>(acc[g % NI][j], fw[g % R], fa[(g / NI) & 1][j]);
            });
            __builtin_amdgcn_sched_barrier(0);
        });
        cs = ns;
    };
    int kt = 0;
    for (const int plain = nk - (chunks ? 1 : 0) - NS; kt < plain; ++kt) step(YES, kt);
    for (; kt < bound; ++kt) step(NO, kt);
    // the last look-ahead reads are on their way into the fragment registers: they pass through the wait
    wait_frag<0>(fw[0]);
    settle_mfma();
    static_for<0, NI * MI>([&](auto pc) __attribute__((always_inline)) { constexpr int p = decltype(pc)::value; hold_acc<false>(acc[p / MI][p % MI]); });
#pragma unroll
    for (int r = 1; r < R; ++r) hold_frag(fw[r]);
#pragma unroll
    for (int j = 0; j < MI; ++j) { hold_frag(fa[0][j]); hold_frag(fa[1][j]); }

    if constexpr (KIND == LIN_ADAPT && BM * BN < 256 * 128) {
        if (!a.in_loop) add_adapters(acc, a, group, row0 + wm * TM, n0 + wn * TN);
    }

    asm volatile("s_barrier" ::: "memory");         // every wave has read its last fragments
    store_wave_tile<MI, NI, KIND, PASS, PITCH, CH>(acc, a, bias + wn * TN, out_at + wm * TM, out0, n0 + wn * ON, smem + wave * (PASS * PITCH));
}

template <int BM, int BN, int NS, int WM, int WN, int KIND> drf_status launch_tile_shape(LinArgs a, hipStream_t st)
{
    constexpr size_t smem = (size_t)NS * (BM + BN) * 128 + BN * 4 + BM * 4;
    static_assert(smem <= 160 * 1024, "LDS of a CU");
    static std::atomic<uint64_t> lds_allowed{ 0 };
    auto kern = linear_tile_kernel<BM, BN, NS, WM, WN, KIND>;
    DRF_HIP(allow_lds(reinterpret_cast<const void*>(kern), (int)smem, lds_allowed));
    const long long most = 1 << 22;                                 // (a launch holds fewer than 2^32 threads)
    for (a.first = 0; a.first < a.tiles; a.first += most) {
        hipLaunchKernelGGL(kern, dim3((unsigned)std::min(most, a.tiles - a.first)), dim3(WM * WN * 64), smem, st, a);
        DRF_HIP(hipGetLastError());
    }
    return DRF_OK;
}

}  // namespace

template <int KIND> drf_status launch_linear_tile(int tile, const LinArgs& a, hipStream_t st)
{
    switch (tile) {
    case 0: return launch_tile_shape<256, 256, 2, 4, 2, KIND>(a, st);
    case 1: return launch_tile_shape<256, 128, 3, 4, 2, KIND>(a, st);
    case 2: return launch_tile_shape<128, 128, 4, 4, 2, KIND>(a, st);
    case 3: return launch_tile_shape<128, 64, 3, 2, 2, KIND>(a, st);
    case 4: return launch_tile_shape<64, 128, 3, 2, 2, KIND>(a, st);
    case 5: return launch_tile_shape<64, 64, 4, 2, 2, KIND>(a, st);
    case 6: return launch_wide_shape<256, KIND>(a, st);
    default:
        if constexpr (KIND == LIN_GLU) DRF_FAIL(DRF_EINVAL, "no such tile");
        else return launch_wide_shape<288, KIND>(a, st);
    }
}

template <typename T, int KIND> drf_status launch_linear_direct(int form, const LinArgs& a, hipStream_t st)
{
    switch (form) {
    case 0: return launch_direct_shape<T, KIND, 1, KIND == LIN_GLU ? 2 : 1, 16, KIND == LIN_GLU ? 2 : 5>(a, st);     // (16 waves: 128 registers a lane)
    case 1:
        if constexpr (sizeof(T) == 2) return launch_direct_shape<T, KIND, 1, 4, 8, 3>(a, st);
        DRF_FAIL(DRF_EINVAL, "no such form");
    case 2: return launch_direct_shape<T, KIND, 2, 2, 8, 3>(a, st);
    case 3: return launch_direct_shape<T, KIND, 4, 2, 8, 2>(a, st);
    case 4: return launch_direct_shape<T, KIND, 1, 2, 8, 4>(a, st);
    default:
        if constexpr (sizeof(T) == 2 && KIND != LIN_GLU) return launch_direct_shape<T, KIND, 1, 1, 16, 2, 2>(a, st);
        DRF_FAIL(DRF_EINVAL, "no such form");
    }
}

}  // namespace drf
