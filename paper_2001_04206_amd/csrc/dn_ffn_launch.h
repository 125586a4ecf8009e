// The launches of the block's matrix products for one type of element; included by the source of each type.
#pragma once

#include "dn_ffn_few.h"

namespace dn {
namespace {

template <class T, int P, int EPI, class S>
hipError_t tiles(ProductArgs &a, bool sums, hipStream_t s)
{
    a.tiles_m = (a.M + S::BM - 1) / S::BM;
    const int cols = EPI == E_GATED ? S::BN / 2 : S::BN;
    a.tiles_n = (a.N + cols - 1) / cols;
    const dim3 grid((unsigned)(a.tiles_m * a.tiles_n), (unsigned)a.split);
    if constexpr (P == P_GRAD && S::TM != 8) {
        if (sums) {
            launch_kernel(product_kernel<T, P, EPI, S, true>, grid, dim3(S::NW * 64), 0, s, a);
            return hipGetLastError();
        }
    }
    launch_kernel(product_kernel<T, P, EPI, S, false>, grid, dim3(S::NW * 64), 0, s, a);
    return hipGetLastError();
}

template <class T, int EPI, int WAVES, bool WHOLE>
hipError_t few_in(const ProductArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.N + 15) / 16)), block(WAVES * 64);
    if (a.M <= 16) launch_kernel(few_kernel<T, EPI, 1, WAVES, WHOLE>, grid, block, 0, s, a);
    else if (a.M <= 32) launch_kernel(few_kernel<T, EPI, 2, WAVES, WHOLE>, grid, block, 0, s, a);
    else if (a.M <= 48) launch_kernel(few_kernel<T, EPI, 3, WAVES, WHOLE>, grid, block, 0, s, a);
    else launch_kernel(few_kernel<T, EPI, 4, WAVES, WHOLE>, grid, block, 0, s, a);
    return hipGetLastError();
}

template <class T, int EPI, bool WHOLE>
hipError_t few_of(const ProductArgs &a, hipStream_t s)
{
    if (a.M <= 4) {
        const dim3 grid((unsigned)((a.N + 7) / 8)), block(256);
        if (a.M == 1) launch_kernel(token_kernel<T, EPI, 1, WHOLE>, grid, block, 0, s, a);
        else if (a.M == 2) launch_kernel(token_kernel<T, EPI, 2, WHOLE>, grid, block, 0, s, a);
        else launch_kernel(token_kernel<T, EPI, 4, WHOLE>, grid, block, 0, s, a);
        return hipGetLastError();
    }
    // with no more workgroups than compute units, twice the waves in each: 8 rows of 8192 by 4096, bf16, 18.3 us (8 waves: 20.5)
    if (a.N <= 16 * 256) return few_in<T, EPI, 16, WHOLE>(a, s);
    return few_in<T, EPI, 8, WHOLE>(a, s);
}

template <class T, int EPI>
hipError_t few(const ProductArgs &a, hipStream_t s)
{
    // whether all rows lie at multiples of 16 bytes and end at some
    uintptr_t all = (uintptr_t)a.a[0] | (uintptr_t)a.b[0] | (uintptr_t)a.b[1] | (uintptr_t)a.lda | (uintptr_t)a.ldb | (uintptr_t)a.K * sizeof(T);
    return all % 16 == 0 ? few_of<T, EPI, true>(a, s) : few_of<T, EPI, false>(a, s);
}

template <class T, int P, int EPI>
hipError_t run(const ProductPlan &plan, ProductArgs &a, hipStream_t s)
{
    bool sums = a.f.sums || a.f.sums2;
    a.split = plan.split;
    a.steps = plan.steps;
    hipError_t e = hipErrorInvalidValue;
    switch (plan.kernel) {
    case K_FEW:
        if constexpr (P == P_FWD) return few<T, EPI>(a, s);
        return hipErrorInvalidValue;
    case K_SMALL:
        e = tiles<T, P, EPI, Small>(a, sums, s);
        break;
    case K_TINY:
        if constexpr (sizeof(T) == 4) e = tiles<T, P, EPI, Tiny>(a, sums, s);
        break;
    case K_MEDIUM:
        if constexpr (sizeof(T) == 2) e = tiles<T, P, EPI, Medium>(a, sums, s);
        break;
    case K_LARGE:
        if constexpr (sizeof(T) == 2) {
            if (P == P_GRAD && sums) {
                ProductArgs b = a;
                if (a.split > 1) b.ws += (int64_t)a.split * a.M * a.N;
                launch_kernel(sum_parts_kernel<T>, dim3((unsigned)((a.M + 255) / 256), kSumParts), dim3(256), 0, s, b);
                launch_kernel(sum_join_kernel<T>, dim3((unsigned)((a.M + 255) / 256)), dim3(256), 0, s, b);
                if ((e = hipGetLastError()) != hipSuccess) return e;
                sums = false;
            }
            e = tiles<T, P, EPI, Large>(a, false, s);
        }
        break;
    }
    if (e != hipSuccess || a.split == 1) return e;
    const int64_t work = (int64_t)a.M * ((a.N + 7) / 8);
    const int64_t threads = sums && work < a.M ? a.M : work;
    launch_kernel(join_kernel<T, EPI>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a, (int)sums);
    return hipGetLastError();
}

}  // namespace

template <class T>
hipError_t launch_product(Product p, Epilogue e, const ProductPlan &plan, ProductArgs &a, hipStream_t s)
{
    switch (p) {
    case P_FWD:
        if (e == E_LINEAR) return run<T, P_FWD, E_LINEAR>(plan, a, s);
        if (e == E_GATED) return run<T, P_FWD, E_GATED>(plan, a, s);
        return hipErrorInvalidValue;
    case P_DELTA:
        if (e == E_DGATED) return run<T, P_DELTA, E_DGATED>(plan, a, s);
        if (e == E_STORE) return run<T, P_DELTA, E_STORE>(plan, a, s);
        return hipErrorInvalidValue;
    default:
        return e == E_STORE ? run<T, P_GRAD, E_STORE>(plan, a, s) : hipErrorInvalidValue;
    }
}

}  // namespace dn
