// What the Newton-Schulz kernels share on the device: units, splits, the momentum.
#pragma once
#include "gvq_muon.h"
#include "gvq_tile.h"

// A from sums of products of X (both in their units, see gvq_muon_plan.h).
#define NS_GRAM_SCALE (1.f / (1 << NS_X_BITS))

__device__ __forceinline__ void split_f16(float v, _Float16& hi, _Float16& lo)
{
    hi = (_Float16)v;
    lo = (_Float16)(v - (float)hi);
}

// Sum over a work-group, in a fixed order; every thread gets it.
template <int THREADS>
__device__ __forceinline__ double group_sum(double v, double* lds)
{
#pragma unroll
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) s += lds[w];
    __syncthreads();
    return s;
}

// From the sum of U's squares: what U is multiplied with to become X in its units.  r: |X|.
__device__ __forceinline__ double scale_to_x(double squares, double eps, double& r)
{
    const double norm = sqrt(squares), inv = 1.0 / (norm + eps);
    r = norm * inv;
    return ldexp(inv, NS_X_BITS + (ns_is_whole(r) ? 0 : ns_unit_x(r)));
}
// The factors of a matrix's steps, by a whole work-group; `to` may be read behind a barrier (or by the next launch).
__device__ __forceinline__ void leave_factors(const MuonCoef& coef, double r, NsFactors* to)
{
    if (ns_is_whole(r)) {
        if (threadIdx.x < coef.steps) to[threadIdx.x] = coef.whole[threadIdx.x];
    } else if (threadIdx.x == 0) {
        ns_factors(coef.v[0], coef.steps, r, to);
    }
}

__device__ __forceinline__ float number_at(const float* g, int64_t i) { return g[i]; }
__device__ __forceinline__ float number_at(const unsigned short* g, int64_t i) { return bf16_to_f32(g[i]); }

__device__ __forceinline__ void four_numbers(const float* p, float (&u)[4])   // from an aligned place
{
    const f4 v = *(const f4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = v[i];
}
__device__ __forceinline__ void four_numbers(const unsigned short* p, float (&u)[4])
{
    const u2 v = *(const u2*)p;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        u[2 * i] = __uint_as_float(v[i] << 16);
        u[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
}

// U at row r and column c as the momentum already is.
template <typename G>
__device__ __forceinline__ float direction_at(const MuonPrep& a, const G* g, int64_t r, int64_t c)
{
    const float u = number_at(g, r * a.ld_grad + c);
    if (!a.momentum) return u;
    const float m = a.momentum[r * a.ld_momentum + c];
    return a.nesterov ? u + a.beta * m : m;
}
// ... and with the momentum brought up to date first: M <- beta M + G.
template <typename G>
__device__ __forceinline__ float momentum_at(const MuonPrep& a, const G* g, int64_t r, int64_t c)
{
    const float u = number_at(g, r * a.ld_grad + c);
    if (!a.momentum) return u;
    float* m = a.momentum + r * a.ld_momentum + c;
    const float v = a.beta * *m + u;
    *m = v;
    return a.nesterov ? u + a.beta * v : v;
}
