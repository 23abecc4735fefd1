// How much of a prompt's attention each of its tokens got: the column sums of the causal softmax, from the queries, the keys and the log of each
// row's sum (the log-sum-exp that the prompt's attention leaves).
//   got[key head][u] = sum over the query heads of the key head and the rows t >= max(u, first_row) of exp(q_t k_u / sqrt(d) - lse_t)
// No softmax state and no second product: one score product by v_mfma_f32_32x32x16_bf16 with the keys as rows, S^T[u][t], the exponential, and a
// sum over t that stays in registers until the last tile.
#include <type_traits>

#include "kernels.h"
#include "tiles.h"

// KW waves side by side own 64 keys each, their fragments in registers for all heads and queries; the 8 / KW groups of such waves take the tiles of
// 32 queries in turn, through LDS, one tile ahead.  A workgroup has key block b and, PAIRED, the one as far from the end, so that all have the same
// number of tiles.
constexpr int AW_WAVES = 8;
template <int DH, int KW, bool DIRECT>
__global__ __launch_bounds__(AW_WAVES * 64, 2) void attn_weights_kernel(const bf16_t* __restrict__ q, long ldq, const bf16_t* __restrict__ k, long ldk, int T,
                                                                        int kv_heads, int group, int first_row, const float* __restrict__ lse,
                                                                        float scale_log2e, const float* w_in, long ldi, float* w_out, long ldo, int n_blocks,
                                                                        int paired) {
    constexpr int QG = AW_WAVES / KW, KB = 64 * KW, NKS = DH / 16, TB = 32 * DH * 2, NI = TB / 1024 / KW;
    static_assert(NI >= 1, "every wave of a group fetches a part of a tile");
    extern __shared__ __align__(16) unsigned char smem_raw[];            // [QG][2] tiles, then a sum for each key and group
    float* red = (float*)(smem_raw + QG * 2 * TB);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, g = lane >> 5;
    const int kw = wave % KW, qg = wave / KW;
    const int head = blockIdx.x % kv_heads, pair = blockIdx.x / kv_heads;
    const unsigned lds0 = (unsigned)(size_t)smem_raw + qg * 2 * TB, row_at = row_frag_at<DH>(lane);
    const TileFetch<DH, DIRECT> fetch_rows(lane);
    const int n_tiles_all = (T + 31) >> 5;
    for (int part = 0; part < 2; ++part) {
        const int block = part ? n_blocks - 1 - pair : pair;
        if (part && (!paired || block <= pair)) break;
        const int u0 = block * KB + kw * 64;                              // the wave's first key
        bf16x8_t kf[2][NKS];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bf16_t* kr = k + (long)min(u0 + 32 * h + l32, T - 1) * ldk + (long)head * DH + g * 8;
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) kf[h][ks] = load_any16(kr + ks * 16);
        }
        float got[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) got[i] = 0.f;
        const int tile0 = max(block * KB, first_row) >> 5, n_tiles = n_tiles_all - tile0, n_items = n_tiles > 0 ? n_tiles * group : 0;
        const int n_iter = (n_items + QG - 1) / QG;
        // item = query head of the group * n_tiles + tile
        int item = qg, j = 0, tile = qg;
        auto settle = [&]() {
            while (tile >= n_tiles && j < group) tile -= n_tiles, ++j;
        };
        float lse_next = 0.f;
        auto fetch = [&](int it) {
            const int jj = min(j, group - 1), t0 = item < n_items ? (tile0 + tile) * 32 : 0, qh = head * group + jj;
            const unsigned at = lds0 + (it & 1) * TB;
#pragma unroll
            for (int i = 0; i < NI; ++i) fetch_rows(q + (long)t0 * ldq + (long)qh * DH, (unsigned)ldq * 2, kw * NI + i, T - 1 - t0, at);
            lse_next = lse[(long)qh * T + min(t0 + l32, T - 1)];
        };
        if (n_iter > 0) {
            settle();
            fetch(0);
        }
        for (int it = 0; it < n_iter; ++it) {
            const int t0 = (tile0 + tile) * 32, t = t0 + l32;
            const bool live = item < n_items && t0 + 31 >= u0;             // (uniform) some query of the tile sees some key of the wave
            const float bias = -1.44269504088896340736f * lse_next;
            item += QG, tile += QG;
            settle();
            wait_vmcnt<0>();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (it + 1 < n_iter) fetch(it + 1);
            if (!live) continue;
            const unsigned char* sq = smem_raw + (qg * 2 + (it & 1)) * TB;
            f32x16_t s0 = zero16(), s1 = zero16();
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) {
                const bf16x8_t b = *(const bf16x8_t*)(sq + (row_at ^ (unsigned)(ks << 5)));
                s0 = mfma32(kf[0][ks], b, s0);
                s1 = mfma32(kf[1][ks], b, s1);
            }
            if (t0 >= u0 + 63 && t0 + 32 <= T && t0 >= first_row) {       // (uniform) every query counts for every key
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    got[v] += __builtin_amdgcn_exp2f(fmaf(s0[v], scale_log2e, bias));
                    got[16 + v] += __builtin_amdgcn_exp2f(fmaf(s1[v], scale_log2e, bias));
                }
            } else {
                const bool row = t < T && t >= first_row;
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int u = u0 + 8 * (v / 4) + 4 * g + v % 4;
                    const float p0 = __builtin_amdgcn_exp2f(fmaf(s0[v], scale_log2e, bias)), p1 = __builtin_amdgcn_exp2f(fmaf(s1[v], scale_log2e, bias));
                    got[v] += row && t >= u ? p0 : 0.f;
                    got[16 + v] += row && t >= u + 32 ? p1 : 0.f;
                }
            }
        }
        // 32 values over 32 lanes: halves exchanged, lane l32 ends up with the sum of value l32
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            const bool up = l32 & off;
#pragma unroll
            for (int i = 0; i < off; ++i) {
                const float keep = up ? got[i + off] : got[i], give = up ? got[i] : got[i + off];
                got[i] = keep + __shfl_xor(give, off, 64);
            }
        }
        __syncthreads();                                                  // (the block before has been read)
        red[qg * KB + kw * 64 + 32 * (l32 >> 4) + 8 * ((l32 & 15) >> 2) + 4 * g + (l32 & 3)] = got[0];
        __syncthreads();
        for (int i = threadIdx.x; i < KB; i += AW_WAVES * 64) {
            const int u = block * KB + i;
            if (u >= T) break;
            float sum = 0.f;
#pragma unroll
            for (int x = 0; x < QG; ++x) sum += red[x * KB + i];
            w_out[(long)head * ldo + u] = (w_in ? w_in[(long)head * ldi + u] : 0.f) + sum;
        }
    }
}
hipError_t launch_attention_weights(const bf16_t* q, long ldq, const bf16_t* k, long ldk, int T, int heads, int kv_heads, int d, int first_row, const float* lse,
                                    const float* w_in, long ldi, float* w_out, long ldo, hipStream_t s) {
    if (T <= 0) return hipSuccess;
    const int group = heads / kv_heads;
    const float scale = 1.44269504088896340736f / sqrtf((float)d);
    // keys side by side share the queries' way to LDS; fewer where the GPU would not be filled
    const int kw = (long)kv_heads * (T / 512) >= 256 ? 4 : (long)kv_heads * (T / 256) >= 256 ? 2 : 1;
    const int n_blocks = cdiv(T, 64 * kw), paired = (long)kv_heads * n_blocks > 512;
    const int grid = kv_heads * (paired ? (n_blocks + 1) / 2 : n_blocks);
    const int groups = AW_WAVES / kw, lds = groups * (2 * 32 * d * 2 + 64 * kw * 4);
    hipError_t e = hipSuccess;
    auto run = [&](auto kernel) {
        e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e == hipSuccess) kernel<<<grid, AW_WAVES * 64, lds, s>>>(q, ldq, k, ldk, T, kv_heads, group, first_row, lse, scale, w_in, ldi, w_out, ldo, n_blocks, paired);
    };
    auto of_kw = [&](auto dh, auto direct) {
        constexpr int DH = decltype(dh)::value;
        constexpr bool DI = decltype(direct)::value;
        if (kw == 4) run(attn_weights_kernel<DH, 4, DI>);
        else if (kw == 2) run(attn_weights_kernel<DH, 2, DI>);
        else run(attn_weights_kernel<DH, 1, DI>);
    };
    using std::integral_constant;
    const bool direct = loads_to_lds(q) && (ldq & 1) == 0;
    if (d == 128) direct ? of_kw(integral_constant<int, 128>{}, integral_constant<bool, true>{}) : of_kw(integral_constant<int, 128>{}, integral_constant<bool, false>{});
    else direct ? of_kw(integral_constant<int, 64>{}, integral_constant<bool, true>{}) : of_kw(integral_constant<int, 64>{}, integral_constant<bool, false>{});
    return e != hipSuccess ? e : hipGetLastError();
}
