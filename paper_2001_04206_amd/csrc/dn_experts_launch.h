// The launches of the experts' products for one type of element; included by the source of each type.
#pragma once

#include "dn_experts.h"
#include "dn_experts_few.h"

namespace dn {
namespace {

template <class T, int P, int EPI, int GROUP, class S>
hipError_t expert_tiles(ProductArgs &a, int64_t tiles, hipStream_t s)
{
    int parts = a.split;
    const int all = (a.K + 128 / (int)sizeof(T) - 1) / (128 / (int)sizeof(T)) * a.segments;
    a.steps = (all + parts - 1) / parts;
    if (S::TM == 8) a.steps = (a.steps + 1) / 2 * 2;   // (its loop takes two at a time)
    a.split = 1;
    const int cols = EPI == E_GATED ? S::BN / 2 : S::BN;
    a.tiles_n = (a.N + cols - 1) / cols;
    constexpr bool TERMS = GROUP == G_TERMS_A || GROUP == G_TERMS_B;
    a.tiles_m = TERMS ? (a.M + S::BM - 1) / S::BM : (int32_t)tiles;
    launch_kernel(product_kernel<T, P, EPI, S, false, GROUP>, dim3((unsigned)a.tiles_m * (unsigned)a.tiles_n, TERMS ? (unsigned)a.group.experts : (unsigned)parts),
                  dim3(S::NW * 64), 0, s, a);
    return hipGetLastError();
}

template <class T, int EPI, int GROUP>
hipError_t expert_few(const ProductArgs &a, int64_t tiles, hipStream_t s)
{
    const uintptr_t all = (uintptr_t)a.a[0] | (uintptr_t)a.b[0] | (uintptr_t)a.b[1] | (uintptr_t)a.lda | (uintptr_t)a.ldb | (uintptr_t)a.group.b_stride |
                          (uintptr_t)a.K * sizeof(T);
    const dim3 grid((unsigned)((a.N + 15) / 16) * (unsigned)tiles);
    // four waves have all of a short k under way, and more workgroups run at once
    const bool shorter = (int64_t)a.K * (int)sizeof(T) <= 4 * 4 * 128;
    if (all % 16 == 0) {
        if (shorter) launch_kernel(experts_few_kernel<T, EPI, 4, true, GROUP>, grid, dim3(256), 0, s, a);
        else launch_kernel(experts_few_kernel<T, EPI, 8, true, GROUP>, grid, dim3(512), 0, s, a);
    } else {
        if (shorter) launch_kernel(experts_few_kernel<T, EPI, 4, false, GROUP>, grid, dim3(256), 0, s, a);
        else launch_kernel(experts_few_kernel<T, EPI, 8, false, GROUP>, grid, dim3(512), 0, s, a);
    }
    return hipGetLastError();
}

template <class T, int P, int EPI, int GROUP>
hipError_t expert_run(ProductKernel kernel, ProductArgs &a, int64_t tiles, hipStream_t s)
{
    if constexpr (P == P_FWD && EPI != E_PAIR)   // (few rows leave pairs' results in fp32)
        if (kernel == K_FEW) return expert_few<T, EPI, GROUP>(a, tiles, s);
    if (kernel == K_SMALL) return expert_tiles<T, P, EPI, GROUP, Small>(a, tiles, s);
    if constexpr (sizeof(T) == 4) {
        if (kernel == K_TINY) return expert_tiles<T, P, EPI, GROUP, Tiny>(a, tiles, s);
    } else {
        if (kernel == K_MEDIUM) return expert_tiles<T, P, EPI, GROUP, Medium>(a, tiles, s);
        if constexpr (EPI != E_DEXPERT)   // (never planned)
            if (kernel == K_LARGE) return expert_tiles<T, P, EPI, GROUP, Large>(a, tiles, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

template <class T>
hipError_t few_down(const FewDown &a, int rows, hipStream_t s)
{
    const uintptr_t all = (uintptr_t)a.h | (uintptr_t)a.w | (uintptr_t)a.ldh | (uintptr_t)a.ldw | (uintptr_t)a.w_stride | (uintptr_t)a.K * sizeof(T);
    const dim3 grid((unsigned)((a.N + 7) / 8) * (unsigned)rows);
    if (all % 16 == 0) launch_kernel(few_down_kernel<T, true>, grid, dim3(512), 0, s, a);
    else launch_kernel(few_down_kernel<T, false>, grid, dim3(512), 0, s, a);
    return hipGetLastError();
}

template <class T>
hipError_t launch_experts(Product p, Epilogue e, ProductKernel kernel, int gathered, ProductArgs &a, int64_t tiles, hipStream_t s)
{
    if (p == P_FWD && e == E_GATED) return expert_run<T, P_FWD, E_GATED, G_TOKENS>(kernel, a, tiles, s);
    if constexpr (sizeof(T) == 2) {
        if (p == P_FWD && e == E_PAIR) return expert_run<T, P_FWD, E_PAIR, G_ROWS>(kernel, a, tiles, s);
        if (p == P_DELTA && e == E_PAIR) return expert_run<T, P_DELTA, E_PAIR, G_ROWS>(kernel, a, tiles, s);
    }
    if (p == P_FWD && e == E_STORE) return expert_run<T, P_FWD, E_STORE, G_ROWS>(kernel, a, tiles, s);
    if (p == P_DELTA && e == E_DEXPERT) return expert_run<T, P_DELTA, E_DEXPERT, G_TOKENS>(kernel, a, tiles, s);
    if (p == P_DELTA && e == E_STORE) return expert_run<T, P_DELTA, E_STORE, G_ROWS>(kernel, a, tiles, s);
    if (p == P_GRAD && e == E_STORE)
        return gathered == 0 ? expert_run<T, P_GRAD, E_STORE, G_TERMS_A>(kernel, a, tiles, s) : expert_run<T, P_GRAD, E_STORE, G_TERMS_B>(kernel, a, tiles, s);
    return hipErrorInvalidValue;
}

}  // namespace dn
