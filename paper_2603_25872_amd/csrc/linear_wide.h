// The tiles of 256 rows by 256 or 288 rows of the weights for products that fill the chip with them: four waves, one a SIMD, each with 128 x 128 or 128 x 144 of
// the tile and a SIMD's whole register file.  What a tile is made of is as in linear_tile.h; the loop is that of the framework's other products of this size: a
// fixed sequence of matrix instructions with at most one LDS read or one copy beside each, both halves of a step double-buffered in registers, two barriers a step
// (a stage is free from slot REL on, the next one is needed from slot LAND on).  65536 x 4608 x 1152: 479 to 515 us on 256 x 288, 1.35 to 1.45 PFLOP/s, bound by the clock under the matrix
// unit; 65536 x 1152 x 3456 441 to 478 us, 1.09 to 1.18, and 455 to 494 with adapters of rank 32, whose step is one more of 18 and has its copies' offsets made anew.
#pragma once
#include "linear_device.h"

namespace drf {

namespace {

constexpr int kAccPieces = 60;                      // accumulators kept in the matrix unit's own register file

template <int BN, int KIND>
__global__ void __launch_bounds__(256, 1) linear_wide_kernel(const LinArgs a)
{
    constexpr int BM = 256, TM = 128, TN = BN / 2, MI = 8, NI = TN / 16, S = MI * NI, RD = MI + NI, GROUP_M = 8;
    constexpr int STAGE = (BM + BN) * 128, NLA = BM / 32, NLW = BN / 32, NL = NLA + NLW;
    constexpr int ON = KIND == LIN_GLU ? TN / 2 : TN, PITCH = ON * 2 + 16, CH = ON / 8, PASS = 32;
    static_assert(KIND != LIN_GLU || BN == 256, "pairs of pieces in a wave");
    extern __shared__ __attribute__((aligned(128))) unsigned char smem[];   // two stages | bias of the tile's weight rows | where its rows go
    float* bias = reinterpret_cast<float*>(smem + 2 * STAGE);
    uint32_t* out_at = reinterpret_cast<uint32_t*>(bias + (BN + 63) / 64 * 64);

    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave & 1, wn = wave >> 1;
    int tm, tn;
    {
        const long long idx = a.first + item_by_xcd(blockIdx.x, gridDim.x);
        const long long per_group = (long long)GROUP_M * a.tiles_n, group = idx / per_group;
        const int in = (int)(idx - group * per_group), first_m = (int)group * GROUP_M;
        const int gsz = a.tiles_m - first_m < GROUP_M ? a.tiles_m - first_m : GROUP_M;
        tm = first_m + in % gsz;
        tn = in / gsz;
    }
    const int group = tm / a.slot_tiles, row0 = (tm - group * a.slot_tiles) * BM, n0 = tn * (KIND == LIN_GLU ? BN / 2 : BN);
    const int nk = (a.K + 63) / 64, chunks = (a.K & 63) / 8;
    const int ad = KIND == LIN_ADAPT && a.in_loop ? __builtin_amdgcn_readfirstlane(adapter_of(a, group)) : -1;
    const int nt = KIND == LIN_ADAPT && ad >= 0 ? nk + a.low_cols / 32 : nk;
    int slot0, token0;
    const bool some = locate_row(a, group, row0, slot0, token0);
    if (a.slot_rows == a.tokens) {
        if (!some) return;                          // the slot ends before this tile
    } else token0 = 0;
    const char* x0 = (const char*)a.x.data + (slot0 * a.x.slot_stride + token0 * a.x.token_stride) * 2;
    char* out0 = (char*)a.out.data + (slot0 * a.out.slot_stride + token0 * a.out.token_stride) * 2;

    // Copies: wave w takes the activation rows [64 w, ..) and the weight rows [w BN / 4, ..) of a step, 8 rows an instruction.
    const int prow = lane >> 3, ppos = lane & 7;
    uint32_t voff[NL], over[2];                     // over[p]: what the copies of rows with (row / 8) % 2 == p go back by in the last step
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int chunk = ppos ^ ((p * 4 + prow / 2) & 7);
        over[p] = chunks && chunk >= chunks ? (uint32_t)(chunk - chunks + 1) * 16u : 0u;
    }
    const bool odd_w = (BN / 32) % 2 && (wave & 1);
    const uint32_t over_w[2] = { odd_w ? over[1] : over[0], odd_w ? over[0] : over[1] };
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int r = (i < NLA ? wave * 64 + i * 8 : wave * (BN / 4) + (i - NLA) * 8) + prow, chunk = ppos ^ ((r / 2) & 7);
        if (i < NLA) {
            int slot, token;
            if (!locate_row(a, group, row0 + r, slot, token)) { slot = slot0; token = token0; }
            voff[i] = (uint32_t)(((slot - slot0) * a.x.slot_stride + (token - token0) * a.x.token_stride) * 2) + (uint32_t)chunk * 16u;
        } else {
            int n = r;
            if constexpr (KIND == LIN_GLU) n = n / 32 * 16 + n % 16;
            n = n0 + n < a.N ? n : a.N - 1 - n0;
            voff[i] = (uint32_t)n * (uint32_t)a.K * 2u + (uint32_t)chunk * 16u;
        }
    }
    const char* w0 = (const char*)a.w + (size_t)n0 * a.K * 2;
    const char* w1 = w0 + (KIND == LIN_GLU ? (size_t)a.N * a.K * 2 : 0);
    const char* low0 = (const char*)a.low + ((size_t)slot0 * a.tokens + row0) * a.low_cols * 4;
    const char* b0 = (const char*)a.b + ((size_t)(ad < 0 ? 0 : ad) * a.N + n0) * a.rank * 2;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(DRF_LDS_AS unsigned char*)smem;
    const uint32_t dst_a = lds0 + (uint32_t)wave * 64u * 128u, dst_w = lds0 + (uint32_t)(BM + wave * (BN / 4)) * 128u;
    // PLAIN: a step of the product whose rows do not end in it
    auto copy_one = [&](auto ic, auto plain_c, int kt, uint32_t so) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value, step = (i < NLA ? i : i - NLA) * 1024;
        const char* base = (i < NLA ? x0 : KIND == LIN_GLU && (i - NLA) / 2 % 2 == 1 ? w1 : w0) + (size_t)kt * 128;
        uint32_t vo = voff[i];
        if constexpr (!decltype(plain_c)::value) {
            if (KIND == LIN_ADAPT && kt >= nk) {
                const int r = (i < NLA ? wave * 64 + i * 8 : wave * (BN / 4) + (i - NLA) * 8) + prow, chunk = ppos ^ ((r / 2) & 7), e = kt - nk;
                if constexpr (i < NLA) {
                    base = low0 + e * 64;
                    vo = (uint32_t)((row0 + r < a.tokens ? r : 0) * a.low_cols * 4 + (chunk & 3) * 16 + (chunk & 4 ? a.low_cols * 2 : 0));
                } else {
                    const int left = (a.rank - 32 * e) / 8, n = n0 + r < a.N ? r : a.N - 1 - n0;
                    base = b0 + e * 64;
                    vo = (uint32_t)(n * a.rank * 2 + ((chunk & 3) < left ? chunk & 3 : left - 1) * 16);
                }
            } else if (chunks && kt == nk - 1) vo -= i < NLA ? over[i & 1] : over_w[(i - NLA) & 1];
        }
        const uint32_t dst = (i < NLA ? dst_a : dst_w) + so;
        asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3" :: "s"(dst), "n"(step), "v"(vo), "s"(base) : "memory", "scc");
    };
    // step kt has landed for every wave: zeros behind the end of its rows, if they end in it
    auto cut = [&](int kt, uint32_t so) __attribute__((always_inline)) {
        const bool low = KIND == LIN_ADAPT && kt >= nk;
        const int from = low ? (a.rank - 32 * (kt - nk)) / 8 : chunks;
        if (low ? from >= 4 : !chunks || kt != nk - 1) return;
        for (int r = tid + (low ? BM : 0); r < BM + BN; r += 256)
            for (int c = from; c < (low ? 4 : 8); ++c) {
                *reinterpret_cast<u32x4*>(smem + so + r * 128 + (c ^ ((r / 2) & 7)) * 16) = (u32x4){ 0, 0, 0, 0 };
                if (low) *reinterpret_cast<u32x4*>(smem + so + r * 128 + ((c + 4) ^ ((r / 2) & 7)) * 16) = (u32x4){ 0, 0, 0, 0 };
            }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };

    f32x4 acc[NI][MI];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < MI; ++j) acc[i][j] = (f32x4){ 0.f, 0.f, 0.f, 0.f };

    u32x4 fa[2][MI], fw[2][NI];
    const int pos0 = (quarter ^ ((l16 >> 1) & 7)) * 16, pos1 = ((4 + quarter) ^ ((l16 >> 1) & 7)) * 16;
    const uint32_t a_row = lds0 + (uint32_t)(wm * TM + l16) * 128u, w_row = lds0 + (uint32_t)(BM + wn * TN + l16) * 128u;
    const uint32_t la0 = a_row + pos0, la1 = a_row + pos1, lw0 = w_row + pos0, lw1 = w_row + pos1;
    auto read_one = [&](auto rc, auto sc, uint32_t aa, uint32_t wa) __attribute__((always_inline)) {
        constexpr int r = decltype(rc)::value, s = decltype(sc)::value;
        if constexpr (r == 0) lds_read16<0>(fw[s][0], wa);
        else if constexpr (r <= MI) lds_read16<(r - 1) * 2048>(fa[s][r - 1], aa);
        else lds_read16<(r - MI) * 2048>(fw[s][r - MI], wa);
    };
    auto hold_set = [&](auto sc) __attribute__((always_inline)) {
        constexpr int s = decltype(sc)::value;
        static_for<0, MI>([&](auto jc) __attribute__((always_inline)) { hold_frag(fa[s][decltype(jc)::value]); });
        static_for<0, NI>([&](auto ic) __attribute__((always_inline)) { hold_frag(fw[s][decltype(ic)::value]); });
    };
    // reads every RSTEP slots; REL, LAND: slots of the two barriers; copies from LFIRST on, one every LSTEP slots, the FIRST_TILE first of them in the step whose stage
    // they fill again, the others in the next
    constexpr int RSTEP = 2, REL = RSTEP * RD + 2, LAND = S + 24 < 2 * S - RSTEP * RD ? S + 24 : 2 * S - RSTEP * RD, LFIRST = REL + 1, LSTEP = 7;
    constexpr int FIRST_TILE = (2 * S - LFIRST + LSTEP - 1) / LSTEP < NL ? (2 * S - LFIRST + LSTEP - 1) / LSTEP : NL;
    static_assert(REL < S && LAND + RSTEP * RD <= 2 * S && LFIRST + (NL - 1) * LSTEP - 2 * S < REL, "schedule");
    auto copies_before = [](int slot) constexpr { return (slot - LFIRST + LSTEP - 1) / LSTEP < NL ? (slot - LFIRST + LSTEP - 1) / LSTEP : NL; };
    auto copy_at = [](int m) constexpr {            // the copy issued at slot m of a step, -1: none
        for (int c = 0; c < NL; ++c)
            if ((LFIRST + c * LSTEP) % (2 * S) == m) return c;
        return -1;
    };
    constexpr auto C0 = std::integral_constant<int, 0>{};
    constexpr auto C1 = std::integral_constant<int, 1>{};
    constexpr std::true_type YES{};
    constexpr std::false_type NO{};

    stage_bias<BN, 4, KIND>(a, bias, n0, wave);
    static_for<0, NL>([&](auto ic) __attribute__((always_inline)) { copy_one(ic, NO, 0, 0); });
    {
        int slot, token;
        const bool live = locate_row(a, group, row0 + tid, slot, token);
        out_at[tid] = live ? (uint32_t)(((slot - slot0) * a.out.slot_stride + (token - token0) * a.out.token_stride) * 2) : 0xffffffffu;
    }
    wait_lgkmcnt<0>();
    if (nt > 1) {
        static_for<0, FIRST_TILE>([&](auto ic) __attribute__((always_inline)) { copy_one(ic, NO, 1, STAGE); });
        wait_vmcnt<FIRST_TILE>();
    } else wait_vmcnt<0>();
    asm volatile("s_barrier" ::: "memory");
    cut(0, 0);
    static_for<0, RD>([&](auto rc) __attribute__((always_inline)) { read_one(rc, C0, la0, lw0); });
    static_for<0, S>([&](auto pc) __attribute__((always_inline)) { constexpr int p = decltype(pc)::value; hold_acc<(p < kAccPieces)>(acc[p / MI][p % MI]); });
    settle_mfma();
    wait_lgkmcnt<0>();
    hold_set(C0);

    // One step: MFMA slots 0 .. S-1 on the first half's fragments, S .. 2S-1 on the second's.
    // PLAIN: so are the copies that it starts.
    auto tile = [&](auto plain_c, auto load_c, auto next_c, int kt, uint32_t so, uint32_t no) __attribute__((always_inline)) {
        constexpr bool LOAD = decltype(load_c)::value, NEXT = decltype(next_c)::value;
        const uint32_t ca1 = la1 + so, cw1 = lw1 + so, na0 = la0 + no, nw0 = lw0 + no;
        static_for<0, 2 * S>([&](auto mc) __attribute__((always_inline)) {
            constexpr int m = decltype(mc)::value, s = m / S, p = m % S;
            if constexpr (m == REL) {
                wait_lgkmcnt<0>();
                hold_set(C1);
                if constexpr (NEXT) asm volatile("s_barrier" ::: "memory");
            }
            if constexpr (m == LAND && NEXT) {
                wait_vmcnt<LOAD ? copies_before(LAND) : 0>();
                asm volatile("s_barrier" ::: "memory");
                if constexpr (!decltype(plain_c)::value) cut(kt + 1, no);
            }
            if constexpr (m < RSTEP * RD && m % RSTEP == 0) read_one(std::integral_constant<int, m / RSTEP>{}, C1, ca1, cw1);
            if constexpr (NEXT && m >= LAND && m < LAND + RSTEP * RD && (m - LAND) % RSTEP == 0) read_one(std::integral_constant<int, (m - LAND) / RSTEP>{}, C0, na0, nw0);
            if constexpr (copy_at(m) >= 0) {
                if constexpr (copy_at(m) < FIRST_TILE) { if constexpr (LOAD) copy_one(std::integral_constant<int, copy_at(m)>{}, plain_c, kt + 2, so); }
                else if constexpr (NEXT) copy_one(std::integral_constant<int, copy_at(m)>{}, plain_c, kt + 1, no);
            }
            constexpr int i = p / MI, j = i & 1 ? MI - 1 - p % MI : p % MI;      // one operand changes per MFMA
            mfma<(i * MI + j < kAccPieces)>(acc[i][j], fw[s][i], fa[s][j]);
        });
        if constexpr (NEXT) { wait_lgkmcnt<0>(); hold_set(C0); }
    };
    uint32_t so = 0;
    int kt = 0;
    for (const int plain = nk - (chunks ? 1 : 0) - 2; kt < plain; ++kt) {
        tile(YES, YES, YES, kt, so, (uint32_t)STAGE - so);
        so = (uint32_t)STAGE - so;
    }
    if (KIND == LIN_ADAPT || chunks) {
        for (; kt + 2 < nt; ++kt) {
            tile(NO, YES, YES, kt, so, (uint32_t)STAGE - so);
            so = (uint32_t)STAGE - so;
        }
    }
    if (kt + 1 < nt) {
        tile(NO, NO, YES, kt, so, (uint32_t)STAGE - so);
        so = (uint32_t)STAGE - so;
    }
    tile(YES, NO, NO, kt, so, (uint32_t)STAGE - so);
    settle_mfma();
    static_for<0, S>([&](auto pc) __attribute__((always_inline)) { constexpr int p = decltype(pc)::value; hold_acc<(p < kAccPieces)>(acc[p / MI][p % MI]); });

    asm volatile("s_barrier" ::: "memory");         // every wave has read its last fragments
    store_wave_tile<MI, NI, KIND, PASS, PITCH, CH>(acc, a, bias + wn * TN, out_at + wm * TM, out0, n0 + wn * ON, smem + wave * (PASS * PITCH));
}

template <int BN, int KIND> drf_status launch_wide_shape(LinArgs a, hipStream_t st)
{
    constexpr size_t smem = (size_t)2 * (256 + BN) * 128 + (BN + 63) / 64 * 256 + 256 * 4;
    static_assert(smem <= 160 * 1024, "LDS of a CU");
    static std::atomic<uint64_t> lds_allowed{ 0 };
    auto kern = linear_wide_kernel<BN, KIND>;
    DRF_HIP(allow_lds(reinterpret_cast<const void*>(kern), (int)smem, lds_allowed));
    const long long most = 1 << 22;                 // (a launch holds fewer than 2^32 threads)
    for (a.first = 0; a.first < a.tiles; a.first += most) {
        hipLaunchKernelGGL(kern, dim3((unsigned)std::min(most, a.tiles - a.first)), dim3(256), smem, st, a);
        DRF_HIP(hipGetLastError());
    }
    return DRF_OK;
}

}  // namespace

}  // namespace drf
