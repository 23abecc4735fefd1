// A key/value cache on pages: tokens of many texts go in, one new token of each attends, heads forget the tokens that got little attention.
//   k, v [n_pages][heads][page][d] bf16; slot j of sequence s lies on page table[s][j / page] at j % page.  page is a power of two from 16 on, so
// that 16 slots that begin at a multiple of 16 lie on one page.
#include <algorithm>
#include <type_traits>

#include "kernels.h"

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int page_of(const Paged& c, int seq, int slot) {        // -1: not there
    const int id = c.table[(long)seq * c.n_table + (slot >> c.shift)];
    return id >= 0 && id < c.n_pages ? id : -1;
}
__device__ __forceinline__ long slot_at(const Paged& c, int id, int head, int slot) {        // of a head's first slot of 16, or any
    return ((((long)id * c.heads + head) << c.shift) + (slot & ((1 << c.shift) - 1))) * c.d;
}

// ---------------------------------------------------------------- append
// One workgroup a row of new tokens: 16 bytes of k and of v a thread at a time.  Bytes bound it from some hundred rows on (2048 rows of 32 heads of 128: 67 MB in and out, 14 us,
// 4.8 TB/s, as a large copy), below that one chain of loads and stores: 1.8 us for a row, 4.6 for 64.
__global__ __launch_bounds__(256) void paged_append_kernel(Paged c, const int* __restrict__ lengths, const bf16_t* __restrict__ k, long ldk,
                                                           const bf16_t* __restrict__ v, long ldv, const int* __restrict__ first_row,
                                                           const int* __restrict__ pos, float* __restrict__ weights, int* __restrict__ positions, long ldw) {
    const int row = blockIdx.x;
    int seq = row, at = 0;
    if (first_row) {                      // the last sequence that begins at or before the row
        int lo = 0, hi = c.n_seqs;        // (first_row[lo] <= row < first_row[hi], if it lies in any)
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first_row[mid] <= row) lo = mid;
            else hi = mid;
        }
        if (first_row[lo] > row || first_row[lo + 1] <= row) return;
        seq = lo, at = row - first_row[lo];
    }
    const long slot = (long)max(lengths[seq], 0) + at;
    if (slot >= (long)c.n_table << c.shift) return;
    if (weights || positions) {
        for (int h = threadIdx.x; h < c.heads && slot < ldw; h += 256) {
            const long i = ((long)seq * c.heads + h) * ldw + slot;
            if (weights) weights[i] = 0.f;
            if (positions) positions[i] = pos ? pos[row] : (int)slot;
        }
    }
    const int id = page_of(c, seq, (int)slot);
    if (id < 0) return;
    const int per = c.d >> 3, n = c.heads * per;
    for (int i = threadIdx.x; i < n; i += 256) {
        const int h = i / per, e = (i - h * per) * 8;
        const any16_t kw = *(const any16_t*)(k + (long)row * ldk + h * c.d + e), vw = *(const any16_t*)(v + (long)row * ldv + h * c.d + e);
        const long to = slot_at(c, id, h, (int)slot) + e;
        *(uint4*)(c.k + to) = make_uint4(kw.w[0], kw.w[1], kw.w[2], kw.w[3]);
        *(uint4*)(c.v + to) = make_uint4(vw.w[0], vw.w[1], vw.w[2], vw.w[3]);
    }
}
hipError_t launch_paged_append(const Paged& c, const int* lengths, const bf16_t* k, long ldk, const bf16_t* v, long ldv, const int* first_row, int n_rows,
                               const int* pos, float* weights, int* positions, long ldw, hipStream_t s) {
    if (n_rows <= 0) return hipSuccess;
    paged_append_kernel<<<n_rows, 256, 0, s>>>(c, lengths, k, ldk, v, ldv, first_row, pos, weights, positions, ldw);
    return hipGetLastError();
}

// ---------------------------------------------------------------- attention of one new token of each sequence
// The query heads that share a key head are columns, 16 to a workgroup; its waves take the workgroup's range of the keys in turn, 32 at a time:
//   S^T[key][column] = K q^T   and   O^T[d][column] += V^T P^T     by v_mfma_f32_16x16x32_bf16
// (lane = 16 g + m:  A: row m, contraction slots 8 g ..;  B: column m, the same slots;  D: column m, rows 4 g .. 4 g + 3).
// A lane's scores are those of keys 4 g .. 4 g + 3 of either 16, and these are the slots that it has to bring as the second product's
// operands, P as it holds it and the values as rows of V: it loads D / 16 neighbouring columns of each of its eight keys, and the matrix
// product t takes the t-th column of every lane (row m of its result is column m D / 16 + t).  So both K and V come straight from memory as
// they lie there, nothing goes through LDS, and nothing is exchanged between lanes but the maximum, and that only where it grows by 2^8.
// Weights are split into two bf16 parts, cut off and rounded, so that they are off by 2^-15 of themselves (the matrix unit has nothing else to do
// here); the second is above 0, so that an infinite value gives an infinity and not 0 times it.
// What bounds it: HBM for long texts (131072 keys of 8 key heads 81 us, 6.6 TB/s; 64 texts of up to 4096, 683 MB, 117 us, 5.8 TB/s), below that the chain at a
// workgroup's start: length, page, keys (3800 keys of 32 heads 13 us for 63 MB).
__device__ __forceinline__ f32x4_t mfma16(bf16x8_t a, bf16x8_t b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
template <int W> struct Words;
template <> struct Words<4> { typedef u32x4_t type; };
template <> struct Words<2> { typedef u32x2_t type; };

constexpr int PAGED_NW = 4, PAGED_STEP = 32;
template <int D, bool SCORES>
__global__ __launch_bounds__(PAGED_NW * 64, 2) void attn_paged_kernel(Paged c, const int* __restrict__ lengths, int max_len, const bf16_t* __restrict__ q, long ldq,
                                                                      int group, float scale_log2e, bf16_t* __restrict__ o, long ldo, PagedWs ws, int range,
                                                                      int n_ranges) {
    constexpr int NW = PAGED_NW, NST = D / 32, NT = D / 16, NV = D / 32, LDP = D + 4;
    typedef typename Words<NV>::type vword_t;
    __shared__ __align__(16) float part[NW][16 * LDP];     // a column's output, maximum and sum, wave by wave
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m16 = lane & 15, g = lane >> 4;
    const int heads = c.heads * group, split = blockIdx.y, seq = blockIdx.z;
    int head = blockIdx.x, c0 = 0;
    if (group > 16) {                                      // (uniform) several tiles of columns to a key head
        const int tiles = (group + 15) >> 4;
        head = blockIdx.x / tiles, c0 = blockIdx.x % tiles * 16;
    }
    const int n_cols = min(16, group - c0);
    const int len = min(max(lengths[seq], 0), max_len), k0 = split * range, kend = min(k0 + range, len);
    if (k0 >= len && split > 0) return;
    const long qh0 = (long)seq * heads + head * group + c0;

    bf16x8_t qf[NST];
    {
        const bf16_t* qr = q + (long)seq * ldq + (long)(head * group + c0 + min(m16, n_cols - 1)) * D + g * 8;
#pragma unroll
        for (int st = 0; st < NST; ++st) qf[st] = load_any16(qr + st * 32);
    }
    f32x4_t oacc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) oacc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    bool any = false;

    const int n_steps = max(0, (kend - k0 - wave * PAGED_STEP + NW * PAGED_STEP - 1) / (NW * PAGED_STEP));
    auto key_of = [&](int i) { return k0 + (i * NW + wave) * PAGED_STEP; };
    int ids = -1;                                          // lane 2 i + t: the page of the wave's 16 keys t of its i-th step of 32 steps
    auto pages = [&](int i0) {
        const int key = key_of(i0 + (lane >> 1)) + (lane & 1) * 16;
        ids = key < kend ? page_of(c, seq, key) : -1;
    };
    u32x4_t kr[2][NST];
    vword_t vr[8];
    const int k_lane = m16 * D + g * 8, v_lane = g * 4 * D + m16 * NT;
    int id[2], id_next[2];
    auto pick = [&](int i) {
        id_next[0] = __builtin_amdgcn_readlane(ids, 2 * (i & 31));
        id_next[1] = __builtin_amdgcn_readlane(ids, 2 * (i & 31) + 1);
    };
    auto keys = [&](int i) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const bf16_t* p = c.k + slot_at(c, max(id_next[t], 0), head, key_of(i) + 16 * t);
#pragma unroll
            for (int st = 0; st < NST; ++st) kr[t][st] = __builtin_nontemporal_load((const u32x4_t*)(p + k_lane + st * 32));
        }
    };
    auto values = [&](int i) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const bf16_t* p = c.v + slot_at(c, max(id_next[t], 0), head, key_of(i) + 16 * t);
#pragma unroll
            for (int e = 0; e < 4; ++e) vr[4 * t + e] = __builtin_nontemporal_load((const vword_t*)(p + v_lane + e * D));
        }
    };
    if (n_steps > 0) {
        pages(0);
        pick(0);
        keys(0);
        values(0);
    }
    for (int i = 0; i < n_steps; ++i) {
        const int key0 = key_of(i);
        id[0] = id_next[0], id[1] = id_next[1];
        f32x4_t s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < NST; ++st) s[t] = mfma16(__builtin_bit_cast(bf16x8_t, kr[t][st]), qf[st], s[t]);
        }
        if (i + 1 < n_steps) {
            if ((i + 1 & 31) == 0) pages(i + 1);
            pick(i + 1);
            keys(i + 1);
        }
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][e & 3] * scale_log2e;
        const bool full = key0 + 32 <= kend && id[0] >= 0 && id[1] >= 0;        // (uniform)
        if (!full) {
            const vword_t none = {};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool there = key0 + 16 * (e >> 2) + 4 * g + (e & 3) < kend && id[e >> 2] >= 0;
                x[e] = there ? x[e] : -INFINITY;
                vr[e] = there ? vr[e] : none;              // (a weight of 0 does not take an infinity or NaN away)
            }
            any |= id[0] >= 0 || (id[1] >= 0 && key0 + 16 < kend);
        } else {
            any = true;
        }
        if constexpr (SCORES) {
            if (m16 < n_cols) {
                float* to = ws.scores + (qh0 + m16) * ws.ld_scores + key0 + 4 * g;
                *(f32x4_t*)to = f32x4_t{x[0], x[1], x[2], x[3]};
                *(f32x4_t*)(to + 16) = f32x4_t{x[4], x[5], x[6], x[7]};
            }
        }
        float top = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
        if (__builtin_amdgcn_ballot_w64(top > m + 8.f)) {
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float mn = fmaxf(m, top), alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= alpha;
#pragma unroll
            for (int t = 0; t < NT; ++t) oacc[t] *= alpha;
        }
        const float base = m == -INFINITY ? 0.f : m;
        u32x4_t hi_w;
        bf16x8_t lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = __builtin_amdgcn_exp2f(x[e] - base);
            l += x[e];
            lo[e] = (__bf16)fmaxf(x[e] - __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u), 0x1p-126f);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) hi_w[e] = __builtin_amdgcn_perm(__float_as_uint(x[2 * e + 1]), __float_as_uint(x[2 * e]), 0x07060302u);
        const bf16x8_t hi = __builtin_bit_cast(bf16x8_t, hi_w);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            u32x4_t w;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[e] = __builtin_amdgcn_perm(vr[2 * e + 1][t >> 1], vr[2 * e][t >> 1], t & 1 ? 0x07060302u : 0x05040100u);
            const bf16x8_t a = __builtin_bit_cast(bf16x8_t, w);
            oacc[t] = mfma16(a, hi, oacc[t]);
            oacc[t] = mfma16(a, lo, oacc[t]);
        }
        if (i + 1 < n_steps) values(i + 1);
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (any && m == -INFINITY) l = NAN;                    // keys, and none whose score is above -infinity: 0 / 0
    if (m16 < n_cols) {
        float* mine = part[wave] + m16 * LDP;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int t = 0; t < NT; t += 4)
                *(f32x4_t*)(mine + (4 * g + r) * NT + t) = f32x4_t{oacc[t][r], oacc[t + 1][r], oacc[t + 2][r], oacc[t + 3][r]};
        if (g == 0) { mine[D] = m; mine[D + 1] = l; }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n_cols * D; i += NW * 64) {
        const int cc = i / D, e = i % D;
        float mt = -INFINITY, lt = 0.f, ot = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) mt = fmaxf(mt, part[w][cc * LDP + D]);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float* p = part[w] + cc * LDP;
            const float a = mt == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(p[D] - mt);
            if (a != 0.f) lt += a * p[D + 1], ot += a * p[e];
        }
        if (n_ranges == 1) o[(long)seq * ldo + (long)(head * group + c0 + cc) * D + e] = f32_to_bf16(lt == 0.f ? 0.f : ot / lt);
        else ws.o[((qh0 + cc) * n_ranges + split) * D + e] = ot;
        if (e == 0 && (SCORES || n_ranges > 1)) ws.ml[(qh0 + cc) * n_ranges + split] = make_float2(mt, lt);
    }
}

// Of a query head's live ranges: lane i < live has its factor 2^(its largest score - the largest of all) in a, every lane what all weigh; returns the largest.
__device__ __forceinline__ float join_ranges(const float2* ml, int live, int lane, float* a, float* sum) {
    const float2 mine = lane < live ? ml[lane] : make_float2(-INFINITY, 0.f);
    const float top = wave_max(mine.x);
    *a = lane >= live ? 0.f : top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mine.x - top);
    *sum = wave_sum(*a != 0.f ? *a * mine.y : 0.f);
    return top;
}
// Behind the ranges: the first n_join workgroups join the outputs, 256 / D query heads each, NR ranges' columns asked for at a time (as a chain of loads 32 ranges take
// 4.6 us, 8 take 4.0), the others add what 1024 slots of a key head got (33 texts of up to 2000, 40 heads over 8: 7 us for both):
//   weights_out[slot] = weights_in[slot] + the sum over the group's query heads of 2^(x - log2 of the sum of weights)
template <int D, int NR>
__global__ __launch_bounds__(256) void paged_join_kernel(Paged c, const int* __restrict__ lengths, int max_len, int group, bf16_t* __restrict__ o, long ldo,
                                                         PagedWs ws, int range, int n_ranges, int n_join, const float* w_in, float* w_out, long ldw, int n_chunks) {
    const int heads = c.heads * group, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((int)blockIdx.x < n_join) {
        const long qh = (long)blockIdx.x * (256 / D) + threadIdx.x / D;
        if (qh >= (long)c.n_seqs * heads) return;
        const int seq = qh / heads, e = threadIdx.x % D, len = min(max(lengths[seq], 0), max_len), live = (len + range - 1) / range;
        const float* part = ws.o + qh * n_ranges * D + e;
        float t[NR], a, sum, ot = 0.f;
        auto fetch = [&](int i0) {
#pragma unroll
            for (int i = 0; i < NR; ++i) t[i] = part[(long)min(i0 + i, n_ranges - 1) * D];
        };
        fetch(0);
        join_ranges(ws.ml + qh * n_ranges, live, lane, &a, &sum);
        for (int i0 = 0; i0 < live; i0 += NR) {
            if (i0) fetch(i0);
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const float ai = __shfl(a, (i0 + i) & 63, 64);
                ot += i0 + i < live && ai != 0.f ? ai * t[i] : 0.f;      // (a range that weighs nothing, or is none, may hold anything)
            }
        }
        o[(long)seq * ldo + qh % heads * D + e] = f32_to_bf16(sum == 0.f ? 0.f : ot / sum);
        return;
    }
    int idx = blockIdx.x - n_join;
    const int chunk = idx % n_chunks, sh = idx / n_chunks, seq = sh / c.heads, head = sh % c.heads;
    const int len = min(max(lengths[seq], 0), max_len), live = (len + range - 1) / range, key = chunk * 1024 + threadIdx.x * 4;
    if (chunk * 1024 >= len) return;
    constexpr int NH = 8;                                  // query heads at a time
    __shared__ float lse[NH];
    const long at = ((long)seq * c.heads + head) * ldw + key;
    float was[4] = {0.f, 0.f, 0.f, 0.f}, got[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (w_in && key + e < len) was[e] = w_in[at + e];
    for (int g0 = 0; g0 < group; g0 += NH) {
        const int n = min(NH, group - g0);
        const long qh = (long)seq * heads + head * group + g0;
        f32x4_t x[NH];
#pragma unroll
        for (int j = 0; j < NH; ++j)
            if (j < n && key < len) x[j] = *(const f32x4_t*)(ws.scores + (qh + j) * ws.ld_scores + key);
        if (g0) __syncthreads();
        for (int j = wave; j < n; j += 4) {
            float a, sum;
            const float top = join_ranges(ws.ml + (qh + j) * n_ranges, live, lane, &a, &sum);
            if (lane == 0) lse[j] = sum == 0.f ? INFINITY : top + __log2f(sum);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NH; ++j) {
            if (j < n) {
#pragma unroll
                for (int e = 0; e < 4; ++e) got[e] += __builtin_amdgcn_exp2f(x[j][e] - lse[j]);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (key + e < len) w_out[at + e] = was[e] + got[e];
}

static size_t round4(size_t n) { return (n + 3) & ~(size_t)3; }
PagedPlan attention_paged_plan(int max_len, int n_seqs, int heads, int kv_heads, int d, bool weights, size_t ws_elems) {
    const int group = heads / kv_heads, unit = PAGED_NW * PAGED_STEP;
    const long groups = (long)n_seqs * kv_heads * ((group + 15) / 16), rows = (long)n_seqs * heads;
    const size_t scores = weights ? (size_t)rows * (size_t)(((long)max_len + 31) & ~31L) : 0;
    const int most = (int)((max_len + unit - 1L) / unit);
    PagedPlan p;
    // Few key heads in all: as many workgroups as CUs; more: four times that, or, as sequences differ in length and the last round of workgroups is
    // seldom full, ranges of 256 (short texts) or 640 keys.  A range alone needs no second launch.  us, by ranges:
    // 131072 keys of 8 key heads 16 / 24 / 32 / 64: 136 / 102 / 89 / 90; 3800 of 32 heads 4 / 8 / 16: 27 / 21 / 21; 8 texts of up to 4000, 8 key heads 4 / 7 / 8 / 16:
    // 27 / 29 / 26 / 25; 64 of up to 4096 1 / 2 / 4 / 7 / 8 / 16 / 32: 130 / 149 / 140 / 120 / 127 / 131 / 146; 16 of up to 16000 8 / 16 / 24 / 32 / 64: 139 / 118 /
    // 113 / 118 / 123; 33 of up to 2000, with weights 1 / 2 / 4 / 8 / 16: 74 / 64 / 58 / 52 / 53; 64 of up to 500 1 / 2 / 4: 23 / 28 / 31.  Ranges of
    // 256 and of 640 keys around the border, 8 key heads: 64 of up to 1500 50 and 51, 2040 68 and 73, 2400 76 and 88, 3000 96 and 89, 4096 128 and 117; 33 with weights, 2000 48 and 55, 2400 54 and 65, 3600 75 and 79.
    int n = 1;
    if (max_len > 512) n = (int)(groups < 64 ? 256 / groups : std::max(1024 / groups, max_len <= 2048 ? ((long)max_len + 255) / 256 : ((long)max_len + 639) / 640));
    n = n > most ? most : n;
    n = n > PAGED_MAX_RANGES ? PAGED_MAX_RANGES : n;
    for (;; --n) {
        if (n < 1) n = 1;
        p.range = (int)(((long)max_len + n - 1) / n + unit - 1) / unit * unit;
        if (p.range < unit) p.range = unit;
        p.n_ranges = (int)((max_len + (long)p.range - 1) / p.range);
        if (p.n_ranges < 1) p.n_ranges = 1;
        const size_t ml = weights || p.n_ranges > 1 ? round4((size_t)rows * p.n_ranges * 2) : 0, part = p.n_ranges > 1 ? (size_t)rows * p.n_ranges * d : 0;
        p.elems = scores + ml + part;
        p.ml_at = scores;
        p.o_at = scores + ml;
        if (p.elems <= ws_elems || n == 1) return p;
    }
}
hipError_t launch_attention_paged(const Paged& c, const int* lengths, int max_len, const bf16_t* q, long ldq, int heads, bf16_t* o, long ldo, const float* w_in,
                                  float* w_out, long ldw, float* ws, const PagedPlan& p, hipStream_t s) {
    const int group = heads / c.heads, tiles = (group + 15) / 16;
    const float scale = 1.44269504088896340736f / sqrtf((float)c.d);
    PagedWs w;
    if (p.elems) {
        w.scores = ws;
        w.ld_scores = ((long)max_len + 31) & ~31L;
        w.ml = (float2*)(ws + p.ml_at);
        w.o = ws + p.o_at;
    }
    const dim3 grid(c.heads * tiles, p.n_ranges, c.n_seqs);
    auto attend = [&](auto kernel) { kernel<<<grid, PAGED_NW * 64, 0, s>>>(c, lengths, max_len, q, ldq, group, scale, o, ldo, w, p.range, p.n_ranges); };
    if (c.d == 128) w_out ? attend(attn_paged_kernel<128, true>) : attend(attn_paged_kernel<128, false>);
    else w_out ? attend(attn_paged_kernel<64, true>) : attend(attn_paged_kernel<64, false>);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!w_out && p.n_ranges == 1)) return e;
    const int n_join = p.n_ranges > 1 ? cdiv((long)c.n_seqs * heads, 256 / c.d) : 0, n_chunks = w_out ? cdiv(max_len, 1024) : 0;
    auto join = [&](auto kernel) {
        kernel<<<n_join + c.n_seqs * c.heads * n_chunks, 256, 0, s>>>(c, lengths, max_len, group, o, ldo, w, p.range, p.n_ranges, n_join, w_in, w_out, ldw, n_chunks);
    };
    if (c.d == 128) p.n_ranges <= 8 ? join(paged_join_kernel<128, 8>) : join(paged_join_kernel<128, 32>);
    else p.n_ranges <= 8 ? join(paged_join_kernel<64, 8>) : join(paged_join_kernel<64, 32>);
    return hipGetLastError();
}

// ---------------------------------------------------------------- eviction
// One workgroup a sequence and key head: which slots stay.  The order: recent tokens, larger weights, lower slots; the budget-th of it is
// found digit by digit (11, 11 and 10 bits) by counts of a key of 32 bits that has the same order: that of the weight, and the largest for what is recent, which
// all stays.  Where the counts of the first digit say that more come first than stay, the keys become those of the order among these (crowded_key), and the count
// begins again.  Kept slots below the budget stay where they are; the
// i-th slot that becomes free there receives the i-th kept one from behind.  The pairs go to ws: [count or ~length][from .., to ..].
__device__ __forceinline__ unsigned order_key(float w) {
    const unsigned u = __float_as_uint(w + 0.f);           // (-0 counts as 0)
    return w != w ? 0u : u & 0x80000000u ? ~u : u | 0x80000000u;
}
// A slot on no page holds nothing and could take nothing: below the budget it stays, behind it goes before all others.
__device__ __forceinline__ unsigned no_page_key(int slot, int budget) { return slot < budget ? 0xffffffffu : 0u; }
// Only what comes first can stay: the recent ones by their weights, all of them before the others.
__device__ __forceinline__ unsigned crowded_key(bool recent, float w) { return recent ? max(order_key(w), 1u) : 0u; }
// (No weight's key reaches this bin of the first digit.)
constexpr int EVICT_FIRST_BIN = 2047;
// the bin, from the last down, in which the count first reaches `need`: *bin, and what of `need` is left for it (hist: BINS counts)
template <int NT, int BINS>
__device__ __forceinline__ void find_from_top(const int* hist, int* sums, int* found, int need, int* bin, int* left) {
    constexpr int N = 2048 / NT;                           // bins a thread (with 1024 bins half the threads have none)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hi = BINS - 1 - N * threadIdx.x;
    int c[N], all = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = hi - i >= 0 ? hist[hi - i] : 0, all += c[i];
    int run = all;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_up(run, off, 64);
        if (lane >= off) run += o;
    }
    if (lane == 63) sums[wave] = run;
    __syncthreads();
    for (int w = 0; w < wave; ++w) run += sums[w];
    run -= all;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (run < need && need <= run + c[i]) found[0] = hi - i, found[1] = need - run;
        run += c[i];
    }
    __syncthreads();
    *bin = found[0];
    *left = found[1];
}
// Up to 32 slots a thread: weights, positions and then keys stay in registers from their one reading on.  Thread t has slots 4 (k NT + t) + e for k < K,
// e = 0 .. 3, as bits 4 k + e of a mask.  32768 slots of 32 heads: 30 us (146 where every pass read them again, with two barriers and three counts over the waves
// for each 1024 slots); what bounds it is one CU a row, its barriers and scans.
template <int NT, int K>
__global__ __launch_bounds__(NT, 4) void evict_select_kernel(Paged c, const int* __restrict__ lengths, int budget, int n_recent, const float* w_in, const int* p_in,
                                                          long ldw, float* w_out, int* p_out, int* __restrict__ ws, long ws_ld) {
    constexpr int NWV = NT / 64;
    __shared__ int hist[2048];
    __shared__ int sums[NWV], counts[K * NWV], found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), seq = blockIdx.x / c.heads;
    const long row = (long)blockIdx.x * ldw;
    int* list = ws + (long)blockIdx.x * ws_ld;
    const int len = (int)min((long)max(lengths[seq], 0), min(ldw, (long)c.n_table << c.shift));
    if (len <= budget) {
        if (tid == 0) list[0] = ~len;
        for (int i = tid; i < len; i += NT) {
            if (w_out != w_in) w_out[row + i] = w_in[row + i];
            if (p_out != p_in) p_out[row + i] = p_in[row + i];
        }
        return;
    }
    f32x4_t w[K];
    i32x4_t p[K];
    int id[K];
    const float* wr = w_in + row;
    const int* pr = p_in + row;
    const int* tr = c.table + (long)seq * c.n_table;
    constexpr int NEVER = -0x7fffffff - 1;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const unsigned i = 4 * (k * NT + tid);
        w[k] = f32x4_t{0.f, 0.f, 0.f, 0.f}, p[k] = i32x4_t{NEVER, NEVER, NEVER, NEVER};
        if (i + 4 <= (unsigned)len) w[k] = *(const f32x4_t*)(wr + i), p[k] = *(const i32x4_t*)(pr + i);
        id[k] = i < (unsigned)len ? tr[i >> c.shift] : -1;
    }
    if ((len & 3) && tid == (len >> 2) % NT) {             // the last slots, fewer than four
        f32x4_t wt = {0.f, 0.f, 0.f, 0.f};
        i32x4_t pt = {NEVER, NEVER, NEVER, NEVER};
        for (int i = len & ~3, e = 0; e < 3; ++e)
            if (i + e < len) wt[e] = wr[i + e], pt[e] = pr[i + e];
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k == (len >> 2) / NT) w[k] = wt, p[k] = pt;
    }
    for (int i = tid; i < 2048; i += NT) hist[i] = 0;
    int newest = -0x7fffffff - 1;
#pragma unroll
    for (int k = 0; k < K; ++k) newest = max(newest, max(max(p[k][0], p[k][1]), max(p[k][2], p[k][3])));
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) newest = max(newest, __shfl_xor(newest, off, 64));
    if (lane == 0) sums[wave] = newest;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < NWV; ++x) newest = max(newest, sums[x]);
    const long border = (long)newest - n_recent;
    unsigned key[K][4];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool there = id[k] >= 0 && id[k] < c.n_pages;
            key[k][e] = !there ? no_page_key(4 * (k * NT + tid) + e, budget) : (long)p[k][e] > border ? 0xffffffffu : order_key(w[k][e]);
        }
    __builtin_amdgcn_sched_barrier(0);
    unsigned prefix = 0;
    int need = budget;                                     // of the slots whose key begins with the prefix, so many stay
    bool crowded = false;                                  // more come first than stay
    auto digit = [&](auto shift_of, auto above_of) {
        constexpr int SHIFT = decltype(shift_of)::value, ABOVE = decltype(above_of)::value, BINS = 1 << (ABOVE - SHIFT);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (4 * (k * NT + tid) + e < len && (ABOVE == 32 || key[k][e] >> (ABOVE & 31) == prefix >> (ABOVE & 31))) atomicAdd(&hist[key[k][e] >> SHIFT & (BINS - 1)], 1);
        __syncthreads();
        int bin;
        find_from_top<NT, BINS>(hist, sums, found, need, &bin, &need);
        prefix |= (unsigned)bin << SHIFT;
        if (SHIFT == 21 && bin == EVICT_FIRST_BIN) {       // (uniform)
            crowded = hist[EVICT_FIRST_BIN] > need;
            __syncthreads();
        }
        if (SHIFT) {
            for (int i = tid; i < 2048; i += NT) hist[i] = 0;
            __syncthreads();
        }
    };
    using std::integral_constant;
    digit(integral_constant<int, 21>{}, integral_constant<int, 32>{});
    if (crowded) {                                         // (uniform; what the keys were made of is read again, so that no registers hold it)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = 4 * (k * NT + tid) + e;
                const bool first = i < len && key[k][e] == 0xffffffffu;
                if (!first || page_of(c, seq, i) >= 0) key[k][e] = crowded_key(first, first ? wr[i] : 0.f);
            }
        prefix = 0, need = budget;
        digit(integral_constant<int, 21>{}, integral_constant<int, 32>{});
    }
    digit(integral_constant<int, 10>{}, integral_constant<int, 21>{});
    digit(integral_constant<int, 0>{}, integral_constant<int, 10>{});
    const int n_equal = hist[prefix & 1023];
    // f(bit, how many bits are set for slots before it) for each set bit; returns how many there are
    auto in_order = [&](unsigned mask, auto&& f) -> int {
        int below[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            int before = 0, all = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned long long b = __ballot(mask >> (4 * k + e) & 1);
                before += __popcll(b & ((1ull << lane) - 1));
                all += __popcll(b);
            }
            below[k] = before;
            if (lane == 0) counts[k * NWV + wave] = all;
            __builtin_amdgcn_sched_barrier(0);             // (the masks of all eight would not fit the registers)
        }
        __syncthreads();
        constexpr int PER = K * NWV / 64 > 0 ? K * NWV / 64 : 1;      // counts a lane, in order
        int c2[PER], mine = 0;
#pragma unroll
        for (int x = 0; x < PER; ++x) c2[x] = lane * PER + x < K * NWV ? counts[lane * PER + x] : 0, mine += c2[x];
        int run = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int o = __shfl_up(run, off, 64);
            if (lane >= off) run += o;
        }
        const int total = __shfl(run, 63, 64);
        run -= mine;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int at = k * NWV + wave;                 // (uniform)
            int base = 0, upto = run;
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                const int here = __shfl(upto, at / PER, 64);
                if (at % PER == x) base = here;
                upto += c2[x];
            }
            int rank = base + below[k];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (mask >> (4 * k + e) & 1) f(4 * k + e, rank++);
        }
        return total;
    };
    unsigned keep = 0, equal = 0;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool there = 4 * (k * NT + tid) + e < len;
            if (there && key[k][e] > prefix) keep |= 1u << (4 * k + e);
            if (there && key[k][e] == prefix) equal |= 1u << (4 * k + e);
        }
    if (n_equal == need) keep |= equal;                    // (uniform)
    else {
        in_order(equal, [&](int bit, int rank) { if (rank < need) keep |= 1u << bit; });
        __syncthreads();
    }
    // slots that become free and, behind them in the order of the slots, as many that move there
    unsigned marked = 0;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 4 * (k * NT + tid) + e;
            if (i < len && (keep >> (4 * k + e) & 1) == (i >= budget)) marked |= 1u << (4 * k + e);
        }
    const int n = in_order(marked, [&](int bit, int rank) { if (rank < ws_ld - 1) list[1 + rank] = 4 * ((bit >> 2) * NT + tid) + (bit & 3); });
    if (tid == 0) list[0] = n >> 1;
    if (w_out == w_in && p_out == p_in) return;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 4 * (k * NT + tid) + e;
            if (i < budget && keep >> (4 * k + e) & 1) {
                if (w_out != w_in) w_out[row + i] = w_in[row + i];
                if (p_out != p_in) p_out[row + i] = p_in[row + i];
            }
        }
}
// The same for any number of slots, which are read again by every pass; the slots that move there lie `most` behind those that become free.  The call for 8 heads: 40000
// slots 149 us, 131072 452; what bounds it is one CU a head, five readings and four barriers to 1024 slots in the last.
constexpr int EVICT_NT = 1024;
__global__ __launch_bounds__(EVICT_NT) void evict_select_long_kernel(Paged c, const int* __restrict__ lengths, int budget, int n_recent, const float* w_in,
                                                                const int* p_in, long ldw, float* w_out, int* p_out, int* __restrict__ ws, long ws_ld) {
    constexpr int NT = EVICT_NT, NWV = NT / 64;
    __shared__ int hist[2048];
    __shared__ int sums[3][NWV];
    __shared__ int found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, seq = blockIdx.x / c.heads;
    const long row = (long)blockIdx.x * ldw;
    int* list = ws + (long)blockIdx.x * ws_ld;
    const int len = (int)min((long)max(lengths[seq], 0), min(ldw, (long)c.n_table << c.shift));
    if (len <= budget) {
        if (tid == 0) list[0] = ~len;
        for (int i = tid; i < len; i += NT) {
            if (w_out != w_in) w_out[row + i] = w_in[row + i];
            if (p_out != p_in) p_out[row + i] = p_in[row + i];
        }
        return;
    }
    int newest = -0x7fffffff - 1;
    for (int i = tid; i < len; i += NT) newest = max(newest, p_in[row + i]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) newest = max(newest, __shfl_xor(newest, off, 64));
    if (lane == 0) sums[0][wave] = newest;
    __syncthreads();
    for (int w = 0; w < NWV; ++w) newest = max(newest, sums[0][w]);
    const long border = (long)newest - n_recent;
    unsigned recent_bits = 0xffffffffu, other_bits = 0xffffffffu;        // (both 0: crowded_key)
    auto key_of = [&](int i) -> unsigned {
        if (page_of(c, seq, i) < 0) return no_page_key(i, budget);
        const unsigned key = order_key(w_in[row + i]);
        return (long)p_in[row + i] > border ? max(key | recent_bits, 1u) : key & other_bits;
    };
    unsigned prefix = 0;
    int need = budget;                                     // of the slots whose key begins with the prefix, so many stay
    for (int d = 0; d < 3; ++d) {
        const int shift = d == 0 ? 21 : d == 1 ? 10 : 0, bins = d == 2 ? 1024 : 2048;
        __syncthreads();
        for (int i = tid; i < 2048; i += NT) hist[i] = 0;
        __syncthreads();
        const int above = d == 0 ? 32 : d == 1 ? 21 : 10;
        for (int i = tid; i < len; i += NT) {
            const unsigned key = key_of(i);
            if (d == 0 || key >> above == prefix >> above) atomicAdd(&hist[key >> shift & (bins - 1)], 1);
        }
        __syncthreads();
        int bin;
        if (d == 2) find_from_top<NT, 1024>(hist, sums[0], found, need, &bin, &need);
        else find_from_top<NT, 2048>(hist, sums[0], found, need, &bin, &need);
        if (d == 0 && bin == EVICT_FIRST_BIN && hist[EVICT_FIRST_BIN] > need) {        // (uniform; once: then no more slots than stay are left in this bin)
            recent_bits = other_bits = 0, need = budget, d = -1;
            continue;
        }
        prefix |= (unsigned)bin << shift;
    }
    // in the order of the slots: equal keys, slots that become free below the budget, kept ones behind it
    int n_equal = 0, n_free = 0, n_move = 0;
    for (int i0 = 0; i0 < len; i0 += NT) {
        const int i = i0 + tid;
        const unsigned key = i < len ? key_of(i) : 0u;
        const bool equal = i < len && key == prefix;
        const unsigned long long below = (1ull << lane) - 1, eq = __ballot(equal);
        __syncthreads();
        if (lane == 0) sums[0][wave] = __popcll(eq);
        __syncthreads();
        int rank = n_equal + __popcll(eq & below);
        for (int w = 0; w < wave; ++w) rank += sums[0][w];
        const bool keep = i < len && (key > prefix || (equal && rank < need));
        const bool free = i < len && i < budget && !keep, move = keep && i >= budget;
        const unsigned long long fr = __ballot(free), mv = __ballot(move);
        if (lane == 0) sums[1][wave] = __popcll(fr), sums[2][wave] = __popcll(mv);
        __syncthreads();
        int f = n_free + __popcll(fr & below), m = n_move + __popcll(mv & below);
        for (int w = 0; w < wave; ++w) f += sums[1][w], m += sums[2][w];
        const long most = (ws_ld - 1) >> 1;
        if (free && f < most) list[1 + f] = i;
        if (move && m < most) list[1 + most + m] = i;
        if (i < budget && keep) {
            if (w_out != w_in) w_out[row + i] = w_in[row + i];
            if (p_out != p_in) p_out[row + i] = p_in[row + i];
        }
        for (int w = 0; w < NWV; ++w) n_equal += sums[0][w], n_free += sums[1][w], n_move += sums[2][w];
    }
    if (tid == 0) list[0] = n_move;
}
// The rows of the pairs, d / 8 lanes each for k and for v, 32 pairs a workgroup at a time, their weights and positions, and the new lengths.  apart: how far behind
// the first free slot of a list the first one that moves lies (0: as many as there are).  Bytes bound it: 118000 pairs of 512 bytes 31.5 us, 3.85 TB/s in and out.
template <int D>
__global__ __launch_bounds__(256) void evict_move_kernel(Paged c, int budget, const int* __restrict__ ws, long ws_ld, long apart, const float* w_in, const int* p_in,
                                                         long ldw, float* w_out, int* p_out, int* __restrict__ lengths_out, int n_chunks) {
    const int sh = blockIdx.x / n_chunks, chunk = blockIdx.x % n_chunks, seq = sh / c.heads, head = sh % c.heads;
    const int* list = ws + (long)sh * ws_ld;
    const int n = list[0];
    if (head == 0 && chunk == 0 && threadIdx.x == 0) lengths_out[seq] = n < 0 ? ~n : budget;
    const int* froms = list + 1 + (apart ? apart : n);
    const long row = (long)sh * ldw;
    constexpr int PER = D >> 3, PAIRS = 128 / PER, U = 32 / PAIRS;      // lanes of a row, pairs at a time, times
    const int which = threadIdx.x / (2 * PER), part = threadIdx.x % (2 * PER);
    bf16_t* at = (part < PER ? c.k : c.v) + part % PER * 8;
    for (long i0 = chunk * 32L; i0 < n; i0 += n_chunks * 32L) {
        int from[U], to[U], a[U], b[U];
        u32x4_t x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long i = min(i0 + u * PAIRS + which, (long)n - 1);        // (behind the last pair: that one again)
            from[u] = froms[i], to[u] = list[1 + i];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) a[u] = page_of(c, seq, from[u]), b[u] = page_of(c, seq, to[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = *(const u32x4_t*)(at + slot_at(c, max(a[u], 0), head, from[u]));
        float w[U];
        int p[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (part == 0) w[u] = w_in[row + from[u]];
            if (part == 1) p[u] = p_in[row + from[u]];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * PAIRS + which >= n) break;
            if (a[u] >= 0 && b[u] >= 0) *(u32x4_t*)(at + slot_at(c, b[u], head, to[u])) = x[u];
            if (part == 0) w_out[row + to[u]] = w[u];
            if (part == 1) p_out[row + to[u]] = p[u];
        }
    }
}
hipError_t launch_paged_evict(const Paged& c, const int* lengths, int budget, int n_recent, const float* w_in, const int* p_in, long ldw, float* w_out,
                              int* p_out, int* lengths_out, int* ws, hipStream_t s) {
    const long cap = (long)c.n_table << c.shift, width = cap < ldw ? cap : ldw;
    const long most = width - budget < budget ? (width - budget > 0 ? width - budget : 0) : budget, ld = 1 + 2 * most;
    const int rows = c.n_seqs * c.heads;
    // Many threads a row, few slots a thread: latency bounds these kernels.  us, 64 sequences of 8 heads and 2112 slots with 256 threads of up to 32 / 16 slots,
    // 512 of 8, 1024 of 4: 25.5 / 20.5 / 18.3 / 17.2 for the call.  By the room for slots, as lengths are not known here: the same with room for 2112 / 32768 / 65536: 22 / 89 / 68.
    auto select = [&](auto kernel, int threads) { kernel<<<rows, threads, 0, s>>>(c, lengths, budget, n_recent, w_in, p_in, ldw, w_out, p_out, ws, ld); };
    if (width <= 1024) select(evict_select_kernel<256, 1>, 256);
    else if (width <= 4096) select(evict_select_kernel<1024, 1>, 1024);
    else if (width <= 8192) select(evict_select_kernel<1024, 2>, 1024);
    else if (width <= 16384) select(evict_select_kernel<1024, 4>, 1024);
    else if (width <= 32768) select(evict_select_kernel<1024, 8>, 1024);
    else select(evict_select_long_kernel, EVICT_NT);
    const long room = (1L << 23) / rows;                   // (fewer than 2^32 threads in a launch; at most 2^21 rows, so 4 and more)
    const int n_chunks = most > 0 ? (int)(cdiv(most, 32) < room ? cdiv(most, 32) : room) : 1;
    auto move = [&](auto kernel) {
        kernel<<<rows * n_chunks, 256, 0, s>>>(c, budget, ws, ld, width <= 32768 ? 0 : most, w_in, p_in, ldw, w_out, p_out, lengths_out, n_chunks);
    };
    if (c.d == 128) move(evict_move_kernel<128>);
    else move(evict_move_kernel<64>);
    return hipGetLastError();
}
