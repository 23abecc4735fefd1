// How much of a prompt's attention each of its tokens got: the column sums of the causal softmax, from the queries, the keys and the log of each
// row's sum (the log-sum-exp that the prompt's attention leaves).
//   got[key head][u] = sum over the query heads of the key head and the rows t >= max(u, first_row) of exp(q_t k_u / sqrt(d) - lse_t)
// No softmax state and no second product: one score product by v_mfma_f32_32x32x16_bf16 with the keys as rows, S^T[u][t], the exponential, and a
// sum over t that stays in registers until the last tile.
// What bounds it: 16 products (512 cycles of the matrix unit) and 96 vector instructions, 32 of them exponentials at half rate (512 cycles), to 64 keys x 32 queries and
// wave; the two overlap to 1.2 of the longer one.  8192 tokens, 32 heads over 8 key heads: 285 us, 965 TFLOP/s (with zeros for data 249: the card lowers its clock under such
// work); 2048 tokens of 32 heads 30 us, of which the blocks' beginnings, masked tiles and ends are two thirds.
#include <type_traits>

#include "kernels.h"
#include "tiles.h"

// KW waves side by side own 64 keys each, their fragments in registers for all heads and queries; the WAVES / KW groups of such waves take the tiles of
// queries (32, or 64 where waves share them and each tile costs a barrier) in turn, through LDS, up to two tiles ahead.  A workgroup has key block b and,
// PAIRED, the one as far from the end, so that all have the same number of tiles.
constexpr int aw_rows(int kw) { return kw == 1 ? 32 : 64; }
constexpr int aw_buffers(int dh, int kw) { return dh == 128 && kw < 4 ? 2 : 3; }      // as many tiles as fit
template <int DH, int KW, int WAVES, bool DIRECT>
__global__ __launch_bounds__(WAVES * 64, 2) void attn_weights_kernel(const bf16_t* __restrict__ q, long ldq, const bf16_t* __restrict__ k, long ldk, int T,
                                                                        int kv_heads, int group, int first_row, const float* __restrict__ lse,
                                                                        float scale_log2e, const float* w_in, long ldi, float* w_out, long ldo, int n_blocks,
                                                                        int paired) {
    constexpr int QG = WAVES / KW, KB = 64 * KW, NKS = DH / 16, ROWS = aw_rows(KW), SUB = ROWS / 32, NB = aw_buffers(DH, KW);
    constexpr int TQ = ROWS * DH * 2, TB = TQ + 256, NI = TQ / 1024 / KW;      // bytes of a tile's queries, and with their lse; fetches a wave
    static_assert(NI >= 1, "every wave of a group fetches a part of a tile");
    extern __shared__ __align__(16) unsigned char smem_raw[];            // [QG][NB] tiles, then a sum for each key and group
    float* red = (float*)(smem_raw + QG * NB * TB);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, g = lane >> 5;
    const int kw = wave % KW, qg = wave / KW;
    const int head = blockIdx.x % kv_heads, pair = blockIdx.x / kv_heads;
    const unsigned lds0 = (unsigned)(size_t)smem_raw + qg * NB * TB, row_at = row_frag_at<DH>(lane);
    const TileFetch<DH, DIRECT> fetch_rows(lane);
    const int n_tiles_all = (T + ROWS - 1) / ROWS;
    unsigned voff[NI];                                                    // of a tile that ends before the last row
#pragma unroll
    for (int i = 0; i < NI; ++i) voff[i] = fetch_rows.offset((unsigned)ldq * 2, kw * NI + i);
    for (int part = 0; part < 2; ++part) {
        const int block = part ? n_blocks - 1 - pair : pair;
        if (part && (!paired || block <= pair)) break;
        const int u0 = block * KB + kw * 64;                              // the wave's first key
        float got[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) got[i] = 0.f;
        const int tile0 = max(block * KB, first_row) / ROWS, n_tiles = n_tiles_all - tile0, n_items = n_tiles > 0 ? n_tiles * group : 0;
        const int n_iter = (n_items + QG - 1) / QG;
        // The tiles from the last one back, each for every query head of the group before the next: workgroups of a key head then go through the queries
        // together, which come from one XCD's L2.  (item, j, tile): the one to be fetched next
        int item = qg, j = qg, tile = n_tiles - 1;
        auto settle = [&]() {
            while (j >= group) j -= group, --tile;
        };
        int t0_at[NB - 1];                                                // of the tiles on their way, the first query (-1: none that counts)
        unsigned put = 0, get = 0;                                        // the buffers that the next tile goes to and comes from
        auto fetch = [&]() __attribute__((always_inline)) {
            const int t0 = item < n_items ? (tile0 + tile) * ROWS : 0, qh = head * group + j;
            const unsigned at = lds0 + put;
            const bf16_t* base = q + (long)t0 * ldq + (long)qh * DH;
            const float* lb = lse + (long)qh * T + t0;
            put = put == (NB - 1) * TB ? 0 : put + TB;
            if (DIRECT && t0 + ROWS <= T) {
#pragma unroll
                for (int i = 0; i < NI; ++i) load_lds16(voff[i], base, __builtin_amdgcn_readfirstlane(at + (kw * NI + i) * 1024));
            } else {
                constexpr int AT_ONCE = DIRECT ? NI : 1;                  // (through registers one by one)
#pragma unroll AT_ONCE
                for (int i = 0; i < NI; ++i) fetch_rows(base, (unsigned)ldq * 2, kw * NI + i, T - 1 - t0, at);
            }
            load_lds4s(4 * min(ROWS == 64 ? lane : l32, T - 1 - t0), lb, __builtin_amdgcn_readfirstlane(at + TQ));      // (by every wave: their loads are counted alike)
#pragma unroll
            for (int i = 0; i + 1 < NB - 1; ++i) t0_at[i] = t0_at[i + 1];
            t0_at[NB - 2] = item < n_items ? t0 : -1;
            item += QG, j += QG;
            settle();
        };
        settle();
        for (int i = 0; i < NB - 1 && i < n_iter; ++i) fetch();
        if (NB > 2 && n_iter < NB - 1) t0_at[0] = t0_at[NB - 2];          // (one tile in all)
        bf16x8_t kf[2][NKS];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bf16_t* kr = k + (long)min(u0 + 32 * h + l32, T - 1) * ldk + (long)head * DH + g * 8;
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) kf[h][ks] = load_any16(kr + ks * 16);
        }
        // (the fragments are waited for here: the compiler would else wait for them in the loop, and with them for the tiles on their way)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) asm volatile("" : "+v"(kf[h][ks]));
        // the scores of a tile while the weights of the one before are formed: the matrix unit has its half of the work done under the other's
        struct Tile { f32x16_t s0, s1; float bias; int t0; const unsigned char* at; };      // 32 queries
        auto add = [&](const Tile& x, int v) __attribute__((always_inline)) {
            got[v] += __builtin_amdgcn_exp2f(fmaf(x.s0[v], scale_log2e, x.bias));
            got[16 + v] += __builtin_amdgcn_exp2f(fmaf(x.s1[v], scale_log2e, x.bias));
            asm volatile("" : "+v"(got[v]), "+v"(got[16 + v]));           // (here and not behind the products)
        };
        auto scores = [&](Tile& x) __attribute__((always_inline)) {
            x.s0 = zero16(), x.s1 = zero16();
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) {
                const bf16x8_t b = *(const bf16x8_t*)(x.at + (row_at ^ (unsigned)(ks << 5)));
                x.s0 = mfma32(kf[0][ks], b, x.s0);
                x.s1 = mfma32(kf[1][ks], b, x.s1);
            }
        };
        // tile `it` has landed everywhere, the one before is read; another is asked for.  (KW 1: a tile is its one wave's.)
        const unsigned char* tile_at = smem_raw;
        int tile_t0 = -1;
        auto arrive = [&](int it) __attribute__((always_inline)) {
            if (it + NB - 2 < n_iter) wait_vmcnt<DIRECT ? (NB - 2) * (NI + 1) : NB - 2>();
            else wait_vmcnt<0>();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if constexpr (KW > 1) __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            tile_at = smem_raw + qg * NB * TB + get;
            get = get == (NB - 1) * TB ? 0 : get + TB;
            tile_t0 = t0_at[0];
            if (it + NB - 1 < n_iter) fetch();
            else {
#pragma unroll
                for (int i = 0; i + 1 < NB - 1; ++i) t0_at[i] = t0_at[i + 1];
            }
        };
        // the 32 queries `part` of the tile that is there; false: none of them counts for a key of the wave (uniform)
        auto take = [&](Tile& x, int part) __attribute__((always_inline)) -> bool {
            x.at = tile_at + part * 32 * DH * 2;
            x.bias = -1.44269504088896340736f * *(const float*)(tile_at + TQ + 4 * (32 * part + l32));
            x.t0 = tile_t0 + 32 * part;
            if (tile_t0 < 0 || x.t0 + 31 < u0 || x.t0 >= T) x.t0 = -1;
            return x.t0 >= 0;
        };
        // every query of x counts for every key of the wave, and some of the next do; i: x's place, in parts of a tile
        auto full_step = [&](const Tile& x, Tile& next, int i, auto part_of_next) __attribute__((always_inline)) {
            constexpr int PART = decltype(part_of_next)::value;
            if (PART == 0) arrive((i + 1) / SUB);
            take(next, PART);
            bf16x8_t b[4];                                                // fragments on their way
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) b[ks] = *(const bf16x8_t*)(next.at + (row_at ^ (unsigned)(ks << 5)));
            next.s0 = zero16(), next.s1 = zero16();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) {
#pragma unroll
                for (int v = 0; v < 16 / NKS; ++v) add(x, ks * (16 / NKS) + v);
                next.s0 = mfma32(kf[0][ks], b[ks & 3], next.s0);
                next.s1 = mfma32(kf[1][ks], b[ks & 3], next.s1);
                if (ks + 4 < NKS) b[ks & 3] = *(const bf16x8_t*)(next.at + (row_at ^ (unsigned)((ks + 4) << 5)));
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto any_step = [&](const Tile& x, Tile& next, int i, auto part_of_next) __attribute__((always_inline)) {
            constexpr int PART = decltype(part_of_next)::value;
            if (i + 1 < n_iter * SUB) {
                if (PART == 0) arrive((i + 1) / SUB);
                if (take(next, PART)) scores(next);
            }
            if (x.t0 < 0) return;
            const int t = x.t0 + l32;
            const bool row = t < T && t >= first_row;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int u = u0 + 8 * (v / 4) + 4 * g + v % 4;
                const float p0 = __builtin_amdgcn_exp2f(fmaf(x.s0[v], scale_log2e, x.bias)), p1 = __builtin_amdgcn_exp2f(fmaf(x.s1[v], scale_log2e, x.bias));
                got[v] += row && t >= u ? p0 : 0.f;
                got[16 + v] += row && t >= u + 32 ? p1 : 0.f;
            }
        };
        if (n_iter > 0) {
            // tiles of this group: `lo` that may end behind the last token, then full ones up to `hi` (the same for all lanes, not for all waves)
            const int least = max(u0 + 63, first_row), n_full = n_tiles_all - (least + ROWS - 1) / ROWS;
            const int lo = T % ROWS ? (group - qg + QG - 1) / QG : 0, hi = (max(n_full, 0) * group - qg + QG - 1) / QG;
            using First = std::integral_constant<int, 0>;
            using Second = std::integral_constant<int, SUB - 1>;
            Tile a, b;
            arrive(0);
            if (take(a, 0)) scores(a);
            for (int i = 0; i < n_iter * SUB; i += 2) {
                for (; i / SUB >= lo && i / SUB + 3 - SUB < hi; i += 2) {
                    full_step(a, b, i, Second{});
                    full_step(b, a, i + 1, First{});
                }
                any_step(a, b, i, Second{});
                if (i + 1 < n_iter * SUB) any_step(b, a, i + 1, First{});
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
        for (int i = threadIdx.x; i < KB; i += WAVES * 64) {
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
    const bool direct = loads_to_lds(q) && (ldq & 1) == 0;
    // Keys side by side share the queries' way to LDS; fewer where the GPU would not be filled.  Four waves, two workgroups to a CU, where the walk over the queries is
    // short: one workgroup's beginning and end pass under the other's walk.  us with 1, 2, 4 waves side by side of 8, and 1, 2 of 4 (heads over key heads):
    // 1024 tokens, 32/32: 19.1, 16.7, 22.9, 13.3, 16.3; 2048, 32/32: 45.7, 33.6, 37.2, 32.1, 29.9; 2048, 32/8: 37.1, 63.1, -, 45.5, -; 4096, 32/32: 129, 100, 83.2, 98.9, 86.4;
    // 4096, 32/8: 89, 123, 215, 101, 149; 8192, 32/8: 322, 292, 429, 314, 348; 777 of 4/4 with heads of 64: 9.2, 12.9, 17.6, 10.5, 13.6
    const long blocks = (long)kv_heads * ((T + 63) / 64);
    const int kw = blocks >= 2048 ? 4 : blocks >= 1024 ? 2 : 1;
    const int waves = kw < 4 && blocks > 256 && (long)T * group <= 4096 ? 4 : 8;
    const int n_blocks = cdiv(T, 64 * kw), paired = (long)kv_heads * n_blocks > 256 * 8 / waves;
    const int grid = kv_heads * (paired ? (n_blocks + 1) / 2 : n_blocks);
    const int groups = waves / kw, lds = groups * (aw_buffers(d, kw) * (aw_rows(kw) * d * 2 + 256) + 64 * kw * 4);
    hipError_t e = hipSuccess;
    auto run = [&](auto kernel) {
        e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e == hipSuccess)
            kernel<<<grid, waves * 64, lds, s>>>(q, ldq, k, ldk, T, kv_heads, group, first_row, lse, scale, w_in, ldi, w_out, ldo, n_blocks, paired);
    };
    auto of_width = [&](auto dh, auto di) {
        constexpr int DH = decltype(dh)::value;
        constexpr bool DI = decltype(di)::value;
        if (waves == 4) kw == 2 ? run(attn_weights_kernel<DH, 2, 4, DI>) : run(attn_weights_kernel<DH, 1, 4, DI>);
        else if (kw == 4) run(attn_weights_kernel<DH, 4, 8, DI>);
        else if (kw == 2) run(attn_weights_kernel<DH, 2, 8, DI>);
        else run(attn_weights_kernel<DH, 1, 8, DI>);
    };
    auto of = [&](auto dh) { direct ? of_width(dh, std::true_type{}) : of_width(dh, std::false_type{}); };
    if (d == 128) of(std::integral_constant<int, 128>{});
    else of(std::integral_constant<int, 64>{});
    return e != hipSuccess ? e : hipGetLastError();
}
