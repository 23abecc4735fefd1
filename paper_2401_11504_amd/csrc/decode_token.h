// What the kernels of a decoded token share (gfx950): the token's q, k and v, the rotation, and a head's share of the output projection's A o.
#pragma once
#include <type_traits>

#include "kernels.h"

__device__ __forceinline__ float dot8(const uint4& w, const float (&b)[8], float acc) {
    float a[8];
    unpack8(w, a);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc += a[e] * b[e];
    return acc;
}

// One piece's share of A x: part[j] = sum over the piece's C columns of a[j, c] x[c], j < r, by NT threads.  C / 8 lanes share a
// row of A (row stride lda, a points at the piece's first column); x is in LDS, zero past the `left` columns that exist.
// av: the first NA rows per thread, row j = thread / (C / 8) + i * (8 NT / C), fetched ahead by the caller.
template <int C, int NT, int NA>
__device__ __forceinline__ void lowrank_part(const bf16_t* a, long lda, int r, const float* x, int left, uint4 (&av)[NA], float* part) {
    constexpr int LPR = C / 8, STEP = NT / LPR;
    const int sub = threadIdx.x % LPR, jj = threadIdx.x / LPR;
    float xv[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) xv[e] = x[sub * 8 + e];
    for (int j0 = 0; j0 < r; j0 += NA * STEP) {
        if (j0) {
#pragma unroll
            for (int i = 0; i < NA; ++i) av[i] = *(const uint4*)(a + (long)min(j0 + jj + i * STEP, r - 1) * lda + min(sub * 8, left - 8));
        }
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            float v = dot8(av[i], xv, 0.f);
#pragma unroll
            for (int off = LPR >> 1; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
            const int j = j0 + jj + i * STEP;
            if (sub == 0 && j < r) part[j] = v;
        }
    }
}

// One head's rows of the token being decoded, formed by NT threads: raw + B h (fp32 sums, rounded to bf16), q into row[0], with `all` k and v into
// row[1] and row[2]; not rotated yet, and not synchronised.  TPR threads per row of the head, each with every TPR-th eight of the row of B.
template <int DH, int NT>
__device__ __forceinline__ void fresh_rows(const DecodeFresh& fresh, int head, bool all, float (&row)[3][DH]) {
    constexpr int TPR = NT / DH;
    const int c = threadIdx.x / TPR, p = threadIdx.x % TPR;
    float v[3] = {0.f, 0.f, 0.f}, raw[3];
#pragma unroll
    for (int x = 0; x < 3; ++x) raw[x] = fresh.raw[(long)x * fresh.d + head * DH + c];
    constexpr int NC = TPR >= 8 ? 1 : 8 / TPR;                        // pieces of eight per thread and trip: 64 of a row
    auto low = [&](auto rows) {               // every load of a trip before the first is used
        constexpr int NR = decltype(rows)::value;
        for (int j0 = 0; j0 < fresh.r; j0 += NC * TPR * 8) {
            uint4 bv[NR][NC];
            float4 ha[NR][NC], hb[NR][NC];
#pragma unroll
            for (int x = 0; x < NR; ++x)
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    const int j = min(j0 + (i * TPR + p) * 8, fresh.r - 8);
                    bv[x][i] = *(const uint4*)(fresh.b + ((long)x * fresh.d + head * DH + c) * fresh.r + j);
                    ha[x][i] = *(const float4*)(fresh.h + x * fresh.r + j);
                    hb[x][i] = *(const float4*)(fresh.h + x * fresh.r + j + 4);
                }
#pragma unroll
            for (int x = 0; x < NR; ++x)
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    const float4 a = ha[x][i], b = hb[x][i];
                    const float hh[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                    v[x] = j0 + (i * TPR + p) * 8 < fresh.r ? dot8(bv[x][i], hh, v[x]) : v[x];
                }
        }
    };
    if (all) low(std::integral_constant<int, 3>{}); else low(std::integral_constant<int, 1>{});
#pragma unroll
    for (int x = 0; x < 3; ++x) {
#pragma unroll
        for (int off = TPR >> 1; off > 0; off >>= 1) v[x] += __shfl_xor(v[x], off, 64);
        if (p == 0) row[x][c] = bf16_to_f32(f32_to_bf16(raw[x] + v[x]));
    }
}
// q and k are rotated with the (cos, sin) pairs of the token's position (RoPE pairs elements i and i + d_head / 2) and rounded to bf16: eight elements.
__device__ __forceinline__ void rope8(const float* mine, const float* other, const float2 (&row)[8], int sub, int lpk, float* out) {
    const bool first = sub < (lpk >> 1);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float2 cs = row[e];
        const float a = first ? mine[e] : other[e], b = first ? other[e] : mine[e];   // a: first-half element of the pair
        out[e] = bf16_to_f32(f32_to_bf16(first ? a * cs.x - b * cs.y : b * cs.x + a * cs.y));
    }
}

// A head's output row, rounded, to memory, and with out.a its share of the output projection's A o (see lowrank_part).
// c: this thread's column; every thread of the workgroup (NT of them) takes part.
template <int DH, int NT, int NA>
__device__ __forceinline__ void head_output(float v, int c, int head, int n_heads, const DecodeOut& out, uint4 (&av)[NA]) {
    __shared__ float so[DH];
    const bf16_t b = f32_to_bf16(v);
    if ((int)threadIdx.x < DH) {
        out.o[(long)head * DH + c] = b;
        so[c] = bf16_to_f32(b);
    }
    if (!out.a) return;
    __syncthreads();
    lowrank_part<DH, NT, NA>(out.a + (long)head * DH, (long)n_heads * DH, out.r, so, DH, av, out.part + (long)head * out.r);
}
template <int DH, int NT, int NA>
__device__ __forceinline__ void head_output_fetch(int head, int n_heads, const DecodeOut& out, uint4 (&av)[NA]) {
    constexpr int LPR = DH / 8;
    if (!out.a) return;
#pragma unroll
    for (int i = 0; i < NA; ++i)
        av[i] = *(const uint4*)(out.a + (long)min((int)threadIdx.x / LPR + i * (NT / LPR), out.r - 1) * n_heads * DH + head * DH +
                                threadIdx.x % LPR * 8);
}
