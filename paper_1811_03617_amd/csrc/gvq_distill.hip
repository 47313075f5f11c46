// Divergence of a teacher's top logits from a student's softmax over all of its logits, for every row, and its gradient.
//
//   p = softmax(a / t) over the row's entries, q = softmax(z / t):  l = w t^2 sum_j p_j (log p_j - log q_j),  dz = w t (q - p).
//
// One pass keeps each thread's largest logit and its sum of powers; the sums are joined, the row is read again and its gradient leaves.
// Powers are of 2, of (z - largest) c with c = log2(e) / t: the difference first, since z c alone may leave fp32 (masks of the type's lowest
// value) and loses bits that the difference keeps.  Bound: memory.
#include "gvq_distill.h"

// Eight neighbouring logits of a row.
__device__ __forceinline__ void distill_load8(const float* p, float (&v)[8])
{
    const f4 a = *(const f4*)p, b = *((const f4*)p + 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
__device__ __forceinline__ void distill_load8(const unsigned short* p, float (&v)[8])
{
    const u4 a = *(const u4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(a[i] << 16);
        v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void distill_store8(float* p, const float (&v)[8])
{
    *(f4*)p = f4{v[0], v[1], v[2], v[3]};
    *((f4*)p + 1) = f4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void distill_store8(unsigned short* p, const float (&v)[8])
{
    *(u4*)p = u4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ float distill_load(const float* p) { return *p; }
__device__ __forceinline__ float distill_load(const unsigned short* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void distill_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void distill_store(unsigned short* p, float v) { *p = (unsigned short)f32_to_bf16_rne(v); }

// Largest z so far and the sum of 2^((z - largest) c).  As long as there is nothing but -inf, `top` is -inf and differences are taken from 0.
struct DistillSum {
    float top, sum;
};
__device__ __forceinline__ float distill_from(float top) { return top == -INFINITY ? 0.f : top; }
__device__ __forceinline__ float distill_power(float z, float from, float c) { return __builtin_amdgcn_exp2f((z - from) * c); }
template <int N>
__device__ __forceinline__ void distill_add(DistillSum& a, const float (&v)[N], float c)
{
    float m = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, v[i]);
    m = fmaxf(a.top, m);
    const float from = distill_from(m);
    float s = a.sum * distill_power(a.top, from, c);
#pragma unroll
    for (int i = 0; i < N; ++i) s += distill_power(v[i], from, c);
    a.sum = s;
    a.top = m;
}

// A row's numbers before the first whole word of 16 bytes.
template <typename T>
__device__ __forceinline__ int distill_head(const T* p, int n)
{
    const int h = (int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(T);
    return h < n ? h : n;
}

template <int THREADS, typename F>
__device__ __forceinline__ float block_all(float v, float* part, F join)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v = join(v, __shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < THREADS / 64; ++i) v = join(v, part[i]);
    return v;
}

// The row's entries: probabilities into p, the student's logits there into z, places into at (-1: absent).  Returns the sum of p log p.
// All of the work-group; false when there are none.
template <int THREADS, typename T>
__device__ __forceinline__ bool distill_entries(const DistillArgs& a, int64_t row, const T* z, float* p, float* zj, int* at, float* part, float& plogp)
{
    float top = -INFINITY, any = 0.f;
    for (int j = threadIdx.x; j < a.n_top; j += THREADS) {
        const int64_t i = a.index[row * a.ld_index + j];
        const bool there = i >= 0 && i < a.vocab;
        at[j] = there ? (int)i : -1;
        float v = -INFINITY;
        if (there) {
            const int64_t e = row * a.ld_top + j;
            v = a.top_bf16 ? bf16_to_f32(((const unsigned short*)a.top)[e]) : ((const float*)a.top)[e];
            zj[j] = distill_load(z + i);
            any = 1.f;
        }
        p[j] = v;
        top = fmaxf(top, v);
    }
    any = block_all<THREADS>(any, part, [](float x, float y) { return fmaxf(x, y); });
    if (any == 0.f) return false;
    top = block_all<THREADS>(top, part, [](float x, float y) { return fmaxf(x, y); });
    float sum = 0.f;
    for (int j = threadIdx.x; j < a.n_top; j += THREADS)
        if (at[j] >= 0) sum += distill_power(p[j], top, a.log2_t);
    sum = block_all<THREADS>(sum, part, [](float x, float y) { return x + y; });
    const float l2 = __builtin_amdgcn_logf(sum);
    float s = 0.f;
    for (int j = threadIdx.x; j < a.n_top; j += THREADS)
        if (at[j] >= 0) {
            const float l = (p[j] - top) * a.log2_t - l2, q = __builtin_amdgcn_exp2f(l);
            p[j] = q;
            if (q != 0.f) s += q * l;   // (0 log 0 is 0)
        }
    plogp = block_all<THREADS>(s, part, [](float x, float y) { return x + y; });
    return true;
}

// One work-group a row.
template <typename T, int THREADS, bool GRAD>
__global__ __launch_bounds__(THREADS) void distill_row_kernel(DistillArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float part[THREADS / 64];
    float *p = (float*)lds, *zj = p + a.n_top;
    int* at = (int*)(zj + a.n_top);
    const int64_t row = blockIdx.x;
    const T* z = (const T*)a.logits + row * a.ld;
    T* g = GRAD ? (T*)a.grad + row * a.ld_grad : nullptr;
    const float w = a.weight ? a.weight[row] : 1.f;
    float plogp;
    if (w == 0.f || !distill_entries<THREADS>(a, row, z, p, zj, at, part, plogp)) {
        if (threadIdx.x == 0) a.loss[row] = 0.f;
        if (GRAD)
            for (int i = threadIdx.x; i < a.vocab; i += THREADS) distill_store(g + i, 0.f);
        return;
    }
    const float c = a.log2_t;
    const int head = distill_head(z, a.vocab), words = (a.vocab - head) / 8, tail = head + 8 * words;
    DistillSum sum = {-INFINITY, 0.f};
    for (int i = threadIdx.x; i < words; i += THREADS) {
        float v[8];
        distill_load8(z + head + 8 * i, v);
        distill_add(sum, v, c);
    }
    for (int i = threadIdx.x; i < head + a.vocab - tail; i += THREADS) {
        const float v[1] = {distill_load(z + (i < head ? i : tail + i - head))};
        distill_add(sum, v, c);
    }
    const float top = block_all<THREADS>(sum.top, part, [](float x, float y) { return fmaxf(x, y); });
    const float from = distill_from(top);
    const float s = block_all<THREADS>(sum.sum * distill_power(sum.top, from, c), part, [](float x, float y) { return x + y; });
    const float l2 = __builtin_amdgcn_logf(s);
    float l = 0.f;
    for (int j = threadIdx.x; j < a.n_top; j += THREADS)
        if (at[j] >= 0 && p[j] != 0.f) l += p[j] * ((zj[j] - from) * c - l2);
    l = block_all<THREADS>(l, part, [](float x, float y) { return x + y; });
    if (threadIdx.x == 0) a.loss[row] = w * a.t * a.t * 0.69314718f * (plogp - l);
    if constexpr (GRAD) {
        const float scale = w * a.t / s;
        const bool same = (((uintptr_t)g ^ (uintptr_t)z) & 15) == 0;
        for (int i = threadIdx.x; i < words; i += THREADS) {
            float v[8];
            distill_load8(z + head + 8 * i, v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = distill_power(v[k], from, c) * scale;
            if (same) distill_store8(g + head + 8 * i, v);
            else
#pragma unroll
                for (int k = 0; k < 8; ++k) distill_store(g + head + 8 * i + k, v[k]);
        }
        for (int i = threadIdx.x; i < head + a.vocab - tail; i += THREADS) {
            const int e = i < head ? i : tail + i - head;
            distill_store(g + e, distill_power(distill_load(z + e), from, c) * scale);
        }
        // the entries' places once more, now that the rest of the row has been written; the first of several entries of one place has
        // the sum of all
        __syncthreads();
        for (int j = threadIdx.x; j < a.n_top; j += THREADS) {
            if (at[j] < 0) continue;
            float sum_p = 0.f;
            bool first = true;
            for (int k = 0; k < a.n_top; ++k)
                if (at[k] == at[j]) {
                    if (k < j) first = false;
                    sum_p += p[k];
                }
            if (first) distill_store(g + at[j], distill_power(zj[j], from, c) * scale - sum_p * (w * a.t));
        }
    }
}

template <typename T, int THREADS>
static int launch_rows(const DistillArgs& a, hipStream_t st)
{
    const unsigned lds = (unsigned)(12 * a.n_top);
    if (a.grad) hipLaunchKernelGGL((distill_row_kernel<T, THREADS, true>), dim3((unsigned)a.rows), dim3(THREADS), lds, st, a);
    else hipLaunchKernelGGL((distill_row_kernel<T, THREADS, false>), dim3((unsigned)a.rows), dim3(THREADS), lds, st, a);
    GVQ_HIP(hipGetLastError());
    return GVQ_OK;
}

int gvq_launch_distill(const DistillArgs& a, gvq_dtype_t dtype, void* workspace, hipStream_t st)
{
    (void)workspace;
    const bool wide = a.vocab > 8192;
    if (dtype == GVQ_BF16) return wide ? launch_rows<unsigned short, 1024>(a, st) : launch_rows<unsigned short, 256>(a, st);
    return wide ? launch_rows<float, 1024>(a, st) : launch_rows<float, 256>(a, st);
}
