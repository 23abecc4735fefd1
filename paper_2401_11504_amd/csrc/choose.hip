// The choice of the next token: how often each token is in a text, and penalties, a bias and a mask on the logits with the greedy choice.
#include "kernels.h"

// ---------------------------------------------------------------- counts
// counts[r][t] = the number of j with tokens[r][j] = t.  A workgroup counts a range of the vocabulary of one row in LDS, so that the row
// is written once and nothing has to be cleared before; ids outside the range (padding too) are passed over.
template <int RANGE, int NT>
__global__ __launch_bounds__(NT) void token_counts_kernel(const int* __restrict__ tokens, long ldt, int n, int vocab, int* __restrict__ counts,
                                                           long ldc) {
    __shared__ __align__(16) int h[RANGE];
    const int first = blockIdx.x * RANGE, size = min(RANGE, vocab - first), tid = threadIdx.x;
    const int* tok = tokens + (long)blockIdx.y * ldt;
    int t[8];                                              // eight tokens a thread on their way at a time
    auto fetch = [&](int i0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = i0 + j * NT + tid < n ? tok[i0 + j * NT + tid] : -1;
    };
    fetch(0);
    for (int i = tid * 4; i < RANGE; i += NT * 4) *(int4*)(h + i) = make_int4(0, 0, 0, 0);
    __syncthreads();
    for (int i0 = 0; i0 < n; i0 += 8 * NT) {
        if (i0) fetch(i0);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (t[j] >= first && t[j] - first < size) atomicAdd(&h[t[j] - first], 1);
    }
    __syncthreads();
    int* out = counts + (long)blockIdx.y * ldc + first;
    for (int i = tid * 4; i < size; i += NT * 4) {           // (rows begin at any multiple of 4 bytes, which wide stores take)
        if (i + 4 <= size) *(int4*)(out + i) = *(const int4*)(h + i);
        else for (int j = i; j < size; ++j) out[j] = h[j];
    }
}
// counts[r][tokens[r][j]] += add: whole numbers, so the order of the additions changes nothing
__global__ __launch_bounds__(256) void token_counts_add_kernel(const int* __restrict__ tokens, long ldt, int n, int vocab, int add,
                                                               int* __restrict__ counts, long ldc) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int t = tokens[(long)blockIdx.y * ldt + i];
    if (t >= 0 && t < vocab) atomicAdd(counts + (long)blockIdx.y * ldc + t, add);
}
hipError_t launch_token_counts(const int* tokens, long ldt, int rows, int n, int vocab, int add, int* counts, long ldc, hipStream_t s) {
    for (int r = 0; r < rows; r += 32768) {                // (the grid's second axis is limited)
        const int m = rows - r < 32768 ? rows - r : 32768;
        const int* t = tokens + (long)r * ldt;
        int* c = counts + (long)r * ldc;
        // wide ranges read the tokens fewer times, narrow ones fill the GPU with few rows; more threads where there are many tokens to a row
        auto set = [&](auto kernel, int range, int threads) { kernel<<<dim3(cdiv(vocab, range), m), threads, 0, s>>>(t, ldt, n, vocab, c, ldc); };
        const bool few = (long)m * cdiv(vocab, 8192) < 256, many = n > 4096;
        if (!add && few) many ? set(token_counts_kernel<1024, 1024>, 1024, 1024) : set(token_counts_kernel<1024, 256>, 1024, 256);
        else if (!add) many ? set(token_counts_kernel<8192, 1024>, 8192, 1024) : set(token_counts_kernel<8192, 256>, 8192, 256);
        else if (n > 0) token_counts_add_kernel<<<dim3(cdiv(n, 256), m), 256, 0, s>>>(t, ldt, n, vocab, add, c, ldc);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---------------------------------------------------------------- choice
// Every step is rounded to fp32 by itself (no fused multiply-add), so that equal logits stay equal whatever else is done to them.
__device__ __forceinline__ float penalised(float x, int count, float bias, const Choose& c) {
    if (count > 0) {
        x = x > 0.f ? __fdiv_rn(x, c.repetition) : __fmul_rn(x, c.repetition);
        x = __fsub_rn(x, __fadd_rn(__fmul_rn((float)count, c.frequency), c.presence));
    }
    return __fadd_rn(x, bias);
}
struct Best {
    float v = -INFINITY;
    int i = 0x7fffffff;
    __device__ __forceinline__ void take(float ov, int oi) {       // the lowest index among equals; NaN is never larger nor equal
        if (ov > v || (ov == v && oi < i)) { v = ov; i = oi; }
    }
};
template <int NT>
__device__ __forceinline__ Best block_best(Best b) {
    __shared__ float bv[NT / 64];
    __shared__ int bi[NT / 64];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const float ov = __shfl_xor(b.v, off, 64);
        const int oi = __shfl_xor(b.i, off, 64);
        b.take(ov, oi);
    }
    if ((threadIdx.x & 63) == 0) { bv[threadIdx.x >> 6] = b.v; bi[threadIdx.x >> 6] = b.i; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) b.take(bv[w], bi[w]);
    return b;
}
// 16 bytes that are read or written once, past the caches: 512 rows of 128000 145 -> 133 us
typedef float f32x4_once_t __attribute__((ext_vector_type(4)));
typedef int i32x4_once_t __attribute__((ext_vector_type(4)));
// Grid x: pieces of a row, y: rows.  One piece a row: the choice; more: its best to ws[(row * pieces + piece) * 2], joined by choose_join_kernel.
// A thread has four tokens at a time, U times, all asked for before the first is used (rows begin at any multiple of 4 bytes, which 16-byte
// accesses take).  piece: a multiple of 4 NT U.
template <int NT, int U>
__global__ __launch_bounds__(NT) void choose_kernel(Choose c, int vocab, int piece, float* __restrict__ ws) {
    const long r = blockIdx.y;
    const int first = blockIdx.x * piece, end = min(vocab, first + piece);
    const float* x = c.logits + r * c.ldl;
    const int* counts = c.counts ? c.counts + r * c.ldc : nullptr;
    const float* bias = c.bias ? c.bias + r * c.ldb : nullptr;
    const unsigned* allowed = c.allowed ? c.allowed + r * c.lda : nullptr;
    float* out = c.out ? c.out + r * c.ldo : nullptr;
    Best b;
    for (int i0 = first; i0 < end; i0 += 4 * NT * U) {
        float4 xv[U], bv[U];
        int4 cv[U];
        unsigned may[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + (u * NT + (int)threadIdx.x) * 4;
            bv[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            cv[u] = make_int4(0, 0, 0, 0);
            may[u] = i < end ? 15u : 0u;
            if (i + 4 <= end) {
                const f32x4_once_t w = __builtin_nontemporal_load((const f32x4_once_t*)(x + i));
                xv[u] = make_float4(w.x, w.y, w.z, w.w);
                if (counts) {
                    const i32x4_once_t n = __builtin_nontemporal_load((const i32x4_once_t*)(counts + i));
                    cv[u] = make_int4(n.x, n.y, n.z, n.w);
                }
                if (bias) bv[u] = *(const float4*)(bias + i);
            } else {                                       // the last tokens of a row
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool in = i + e < end;
                    (&xv[u].x)[e] = in ? x[i + e] : 0.f;
                    if (counts && in) (&cv[u].x)[e] = counts[i + e];
                    if (bias && in) (&bv[u].x)[e] = bias[i + e];
                }
            }
            if (allowed && i < end) may[u] = allowed[i >> 5] >> (i & 31) & 15u;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + (u * NT + (int)threadIdx.x) * 4;
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool ok = may[u] >> e & 1;
                y[e] = ok ? penalised((&xv[u].x)[e], (&cv[u].x)[e], (&bv[u].x)[e], c) : -INFINITY;
                if (ok && i + e < end) b.take(y[e], i + e);
            }
            if (out && i + 4 <= end) __builtin_nontemporal_store(f32x4_once_t{y[0], y[1], y[2], y[3]}, (f32x4_once_t*)(out + i));
            else if (out) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i + e < end) out[i + e] = y[e];
            }
        }
    }
    if (!c.choice) return;
    b = block_best<NT>(b);
    if (threadIdx.x) return;
    if (!ws) c.choice[r] = b.i == 0x7fffffff ? -1 : b.i;
    else {
        ws[(r * gridDim.x + blockIdx.x) * 2] = b.v;
        ws[(r * gridDim.x + blockIdx.x) * 2 + 1] = __int_as_float(b.i);
    }
}
__global__ __launch_bounds__(64) void choose_join_kernel(const float* __restrict__ ws, int pieces, int* __restrict__ choice) {
    Best b;
    for (int i = threadIdx.x; i < pieces; i += 64) b.take(ws[((long)blockIdx.x * pieces + i) * 2], __float_as_int(ws[((long)blockIdx.x * pieces + i) * 2 + 1]));
    b = block_best<64>(b);
    if (threadIdx.x == 0) choice[blockIdx.x] = b.i == 0x7fffffff ? -1 : b.i;
}
hipError_t launch_choose(const Choose& c, int rows, int vocab, float* ws, size_t ws_elems, hipStream_t s) {
    for (int r = 0; r < rows; r += 32768) {
        const int m = rows - r < 32768 ? rows - r : 32768;
        Choose p = c;
        p.logits += (long)r * c.ldl;
        if (p.counts) p.counts += (long)r * c.ldc;
        if (p.bias) p.bias += (long)r * c.ldb;
        if (p.allowed) p.allowed += (long)r * c.lda;
        if (p.out) p.out += (long)r * c.ldo;
        if (p.choice) p.choice += r;
        // pieces that fill the GPU (1 row of 32000: 13.3 us with one workgroup, 5.6 in pieces and joined; 512 of 128000 162 and 133)
        const int piece = (long)m * vocab < 1 << 19 ? 1024 : 4096, pieces = cdiv(vocab, piece);
        if (ws && pieces > 1 && (size_t)m * pieces * 2 <= ws_elems) {
            if (piece == 1024) choose_kernel<256, 1><<<dim3(pieces, m), 256, 0, s>>>(p, vocab, piece, ws);
            else choose_kernel<256, 4><<<dim3(pieces, m), 256, 0, s>>>(p, vocab, piece, ws);
            if (p.choice) choose_join_kernel<<<m, 64, 0, s>>>(ws, pieces, p.choice);
        } else {
            choose_kernel<1024, 2><<<dim3(1, m), 1024, 0, s>>>(p, vocab, cdiv(vocab, 8192) * 8192, nullptr);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
