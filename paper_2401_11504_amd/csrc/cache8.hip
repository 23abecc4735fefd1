// The key/value cache held in 8 bits, and attention over it (generation side).
//
// A block is 64 consecutive tokens.  Once complete it is stored, head by head, as int8 codes with one fp32 scale for its keys and one
// for its values:  scale = max(largest magnitude, 2^-100) / 127,  code = value / scale rounded to the nearest, ties to even.  The
// tokens of the block that is not complete yet stay bf16 in the tail, so what the cache holds is a function of the tokens alone, not
// of the calls that they arrived in, and no value is ever rounded twice.
// Keys lie as [block][head][D / 64][64 tokens][64 columns], values as [block][head][D][64 tokens] (transposed): both are contiguous
// 1 KB runs for a wave that loads matrix operands of 16 codes a lane straight from memory, and neither has to be transposed there.
#include <algorithm>
#include <type_traits>

#include "decode_token.h"
#include "tiles.h"

static constexpr float kLeastMagnitude = 7.888609052210118e-31f;   // 2^-100: keeps the scale and its reciprocal normal numbers

// x / s rounded to the nearest integer, ties to even, exactly, for |x| <= 127 s (1 + 2^-24) and `inv` within a few ulp of 1 / s:
// x * inv is off by far less than 1, so its rounding n is the answer or next to it, and the remainder x - n s is exact in fp32 (x is a
// bf16 of at least s / 2, a multiple of s's last place; the remainder is below s).
__device__ __forceinline__ int code8(float x, float s, float inv) {
    const float n = rintf(x * inv);
    const float r = fmaf(-n, s, x), half = 0.5f * s;
    const int i = (int)n, odd = i & 1;
    const int up = r > half || (r == half && odd), down = r < -half || (r == -half && odd);
    return i + up - down;
}

// A workgroup of 2 D threads shares a tile of 64 tokens of one head; a thread has 8 columns of 4 consecutive tokens, in 16-byte pieces of a row.
template <int D>
struct Cache8Tile {
    static constexpr int CPR = D / 8, NT = 2 * D;
    static_assert(NT / CPR == 16, "16 groups of 4 tokens");
};
constexpr int VP = 17;      // words of a value row (64 codes) in LDS: odd, so that rows begin in different banks

// One workgroup for a block that the new tokens complete and a head's keys or values (block by block, the heads' keys before their
// values).  Those of the first block also put the rows behind the last complete block into the tail, after they have read the tail.
// exact.k set: the blocks that are completed go there as they came as well.
// Values are turned round through LDS, as codes, four tokens to a word.  Bytes bound it from some 10^4 tokens of 32 heads of 128 on (32768: 160 to 190 us, 4.2
// to 5 TB/s in and out); 333 tokens take 6.4 to 7.2 us, one 2.5: two round trips to memory.
template <int D>
__global__ __launch_bounds__(2 * D) void cache8_append_kernel(Cache8 c, int n_cached, const bf16_t* __restrict__ k, long ldk,
                                                              const bf16_t* __restrict__ v, long ldv, int n_new, Cache8Exact exact) {
    using T = Cache8Tile<D>;
    __shared__ int red[4];
    __shared__ unsigned sv[D * VP];
    const int tid = threadIdx.x, at = blockIdx.x % (2 * c.heads), nth = blockIdx.x / (2 * c.heads);
    const bool values = at >= c.heads;
    const int head = values ? at - c.heads : at;
    const int end = n_cached + n_new, b1 = end >> 6, block = (n_cached >> 6) + nth;
    const int col = tid % T::CPR * 8, t0 = tid / T::CPR * 4;
    const bf16_t* src = (values ? v : k) + (long)head * D + col;
    const long ld = values ? ldv : ldk;
    bf16_t* tail = (values ? c.vt : c.kt) + (long)head * 64 * D;
    bf16_t* k_slot = tail + (col >> 6) * 4096 + t0 * 64 + (col & 63);       // keys: token t0, the thread's columns; a token further: + 64
    bf16_t* v_slot = tail + col * 64 + t0;                                  // values: the thread's tokens, its first column; a column further: + 64
    // the rows of the block that stays incomplete: on their way before anything else is done
    const int base = b1 << 6, lo = max(n_cached, base);
    uint4 rest[4];
    if (nth == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (base + t0 + i >= lo && base + t0 + i < end) rest[i] = *(const uint4*)(src + (long)(base + t0 + i - n_cached) * ld);
    }
    if (block < b1) {
        const int first = block << 6;
        uint4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (first + t0 + i >= n_cached) x[i] = *(const uint4*)(src + (long)(first + t0 + i - n_cached) * ld);
        if (first + t0 < n_cached) {                       // some of its tokens are in the tail
            if (!values) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (first + t0 + i < n_cached) x[i] = *(const uint4*)(k_slot + 64 * i);
            } else {
                uint2 w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = *(const uint2*)(v_slot + 64 * e);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (first + t0 + i < n_cached) {
                        auto get = [&](int e) { return ((i < 2 ? w[e].x : w[e].y) >> 16 * (i & 1)) & 0xffffu; };
                        x[i] = make_uint4(get(0) | get(1) << 16, get(2) | get(3) << 16, get(4) | get(5) << 16, get(6) | get(7) << 16);
                    }
            }
        }
        if (exact.k) {                                     // (uniform) the block as it came as well
            bf16_t* to = (values ? exact.v : exact.k) + ((long)(block - exact.first) * c.heads + head) * 64 * D;
            if (!values) {
#pragma unroll
                for (int i = 0; i < 4; ++i) *(uint4*)(to + (col >> 6) * 4096 + (t0 + i) * 64 + (col & 63)) = x[i];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {              // four tokens of a column
                    const unsigned sel = e & 1 ? 0x07060302u : 0x05040100u;
                    auto pair = [&](int i) { return __builtin_amdgcn_perm((&x[i + 1].x)[e >> 1], (&x[i].x)[e >> 1], sel); };
                    *(uint2*)(to + (col + e) * 64 + t0) = make_uint2(pair(0), pair(2));
                }
            }
        }
        int amax = 0;                                      // bf16 bits of the largest magnitude
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned w = (&x[i].x)[e];
                amax = max(amax, max((int)(w & 0x7fff), (int)(w >> 16 & 0x7fff)));
            }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) amax = max(amax, __shfl_xor(amax, off, 64));
        if ((tid & 63) == 0) red[tid >> 6] = amax;
        __syncthreads();                                   // (and every thread has what it needs of the tail)
#pragma unroll
        for (int w = 0; w < T::NT / 64; ++w) amax = max(amax, red[w]);
        // a value that is not finite has no code: the scale is NaN, and so is everything read through it
        const bool fine = amax < 0x7f80;
        const float s = fine ? fmaxf(__uint_as_float((unsigned)amax << 16), kLeastMagnitude) / 127.f : __builtin_nanf(""), inv = 1.f / s;
        if (tid == 0) (values ? c.vs : c.ks)[(long)block * c.heads + head] = s;
        const long tile = ((long)block * c.heads + head) * 64 * D;
        unsigned q[4][2];                                  // token by token
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float f[8];
            unpack8(x[i], f);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                unsigned w = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) w |= (unsigned)(code8(f[4 * h + e], s, inv) & 255) << 8 * e;
                q[i][h] = fine ? w : 0;
            }
        }
        if (!values) {
#pragma unroll
            for (int i = 0; i < 4; ++i) *(uint2*)(c.k + tile + (col >> 6) * 4096 + (t0 + i) * 64 + (col & 63)) = make_uint2(q[i][0], q[i][1]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {                  // byte e % 4 of the four tokens' words
                const unsigned sel = 0x0c0c0400u + 0x0101u * (e & 3);
                const unsigned lo2 = __builtin_amdgcn_perm(q[1][e >> 2], q[0][e >> 2], sel), hi2 = __builtin_amdgcn_perm(q[3][e >> 2], q[2][e >> 2], sel);
                sv[(col + e) * VP + (t0 >> 2)] = lo2 | hi2 << 16;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int p = i * T::NT + tid;             // 16 bytes of the tile
                const unsigned* w = sv + (p >> 2) * VP + (p & 3) * 4;
                *(uint4*)(c.v + tile + p * 16) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
    if (nth > 0 || base + t0 + 3 < lo || base + t0 >= end) return;
    if (!values) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (base + t0 + i >= lo && base + t0 + i < end) *(uint4*)(k_slot + 64 * i) = rest[i];
    } else {
        uint2 w[8];                                        // the thread's four tokens as they are, the new ones put in
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = *(const uint2*)(v_slot + 64 * e);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (base + t0 + i >= lo && base + t0 + i < end) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const unsigned u = (&rest[i].x)[e >> 1] >> 16 * (e & 1) & 0xffffu;
                    unsigned& old = i < 2 ? w[e].x : w[e].y;
                    old = i & 1 ? (old & 0xffffu) | u << 16 : (old & 0xffff0000u) | u;
                }
            }
#pragma unroll
        for (int e = 0; e < 8; ++e) *(uint2*)(v_slot + 64 * e) = w[e];
    }
}
hipError_t launch_cache8_append(const Cache8& c, int n_cached, const bf16_t* k, long ldk, const bf16_t* v, long ldv, int n_new,
                                hipStream_t s, const Cache8Exact& exact) {
    // at most 2^19 tokens a launch, for the grid's sake; the cache does not depend on where a text is cut
    for (int i = 0; i < n_new;) {
        const int m = min(n_new - i, 1 << 19), at = n_cached + i, done = ((at + m) >> 6) - (at >> 6);
        const int grid = 2 * c.heads * (done > 1 ? done : 1);
        const bf16_t *ki = k + (long)i * ldk, *vi = v + (long)i * ldv;
        if (c.d == 128) cache8_append_kernel<128><<<grid, 256, 0, s>>>(c, at, ki, ldk, vi, ldv, m, exact);
        else cache8_append_kernel<64><<<grid, 128, 0, s>>>(c, at, ki, ldk, vi, ldv, m, exact);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        i += m;
    }
    return hipSuccess;
}

// Tokens first .. first + n - 1 of a cache that holds n_cached as fp32 rows: code * scale (one rounding), the tail's widened.  A thread
// writes 4 columns of a row at a time, past the caches; values are turned round through LDS, as codes.  Bytes bound it: 32768 tokens of 32 heads of
// 128 228 us, 5.9 TB/s in and out (ordinary stores 242; column pairs straight from memory 620).
template <int D>
__global__ __launch_bounds__(2 * D) void cache8_read_kernel(Cache8 c, int n_cached, int first, int n, float* __restrict__ k, long ldk,
                                                            float* __restrict__ v, long ldv) {
    constexpr int NT = 2 * D, CPR = D / 4, NP = 64 * CPR / NT;              // pieces of 4 columns: a row, a thread
    __shared__ unsigned sv[D * VP];
    const int tid = threadIdx.x, at = blockIdx.x % (2 * c.heads), block = (first >> 6) + blockIdx.x / (2 * c.heads);
    const bool values = at >= c.heads, in_tail = block == n_cached >> 6;
    const int head = values ? at - c.heads : at, row0 = (block << 6) - first;
    const long tile = ((long)block * c.heads + head) * 64 * D;
    const bf16_t* tail = (values ? c.vt : c.kt) + (long)head * 64 * D;
    const int col = tid % CPR * 4, t0 = tid / CPR;                          // 8 token groups
    float* out = (values ? v : k) + (long)head * D + col;
    const long ld = values ? ldv : ldk;
    auto put = [&](int t, float a, float b, float e, float f) {
        const int row = row0 + t;
        if (row >= 0 && row < n) __builtin_nontemporal_store(f32x4_t{a, b, e, f}, (f32x4_t*)(out + (long)row * ld));
    };
    if (in_tail) {
        for (int t = t0; t < 64; t += 8) {
            if (row0 + t < 0 || row0 + t >= n) continue;
            const bf16_t* p = values ? tail + col * 64 + t : tail + (col >> 6) * 4096 + t * 64 + (col & 63);
            const int step = values ? 64 : 1;
            put(t, bf16_to_f32(p[0]), bf16_to_f32(p[step]), bf16_to_f32(p[2 * step]), bf16_to_f32(p[3 * step]));
        }
        return;
    }
    const float s = (values ? c.vs : c.ks)[(long)block * c.heads + head];
    auto value = [&](unsigned w, int e) { return (float)(int8_t)(w >> 8 * e) * s; };
    if (!values) {
        unsigned w[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) w[i] = *(const unsigned*)(c.k + tile + (col >> 6) * 4096 + (t0 + 8 * i) * 64 + (col & 63));
#pragma unroll
        for (int i = 0; i < NP; ++i) put(t0 + 8 * i, value(w[i], 0), value(w[i], 1), value(w[i], 2), value(w[i], 3));
        return;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int p = i * NT + tid;
        const uint4 w = *(const uint4*)(c.v + tile + p * 16);
        unsigned* to = sv + (p >> 2) * VP + (p & 3) * 4;
        to[0] = w.x, to[1] = w.y, to[2] = w.z, to[3] = w.w;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {                                          // four tokens of the thread's columns
        const int tg = t0 + 8 * i;
        unsigned w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = sv[(col + j) * VP + tg];
#pragma unroll
        for (int e = 0; e < 4; ++e) put(tg * 4 + e, value(w[0], e), value(w[1], e), value(w[2], e), value(w[3], e));
    }
}
hipError_t launch_cache8_read(const Cache8& c, int n_cached, int first, int n, float* k, long ldk, float* v, long ldv, hipStream_t s) {
    for (int i = 0; i < n;) {
        const int at = first + i, m = min(n - i, (1 << 19) - (at & 63));      // pieces end where blocks do
        const int grid = 2 * c.heads * (((at + m - 1) >> 6) - (at >> 6) + 1);
        float *ki = k + (long)i * ldk, *vi = v + (long)i * ldv;
        if (c.d == 128) cache8_read_kernel<128><<<grid, 256, 0, s>>>(c, n_cached, at, m, ki, ldk, vi, ldv);
        else cache8_read_kernel<64><<<grid, 128, 0, s>>>(c, n_cached, at, m, ki, ldk, vi, ldv);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        i += m;
    }
    return hipSuccess;
}

// ---------------------------------------------------------------- attention of a few rows
// A row of queries and one of the query heads that share a key head make a column; a workgroup has the columns of one key head (up to 16 with four
// waves, up to 8 with eight), and each of its waves takes every fourth (eighth) block of the workgroup's range of the cache:
//   S^T[key][column] = K q^T   and   O^T[d][column] += V^T P^T     by v_mfma_f32_16x16x32_bf16
// (lane = 16 g + m:  A: row m, contraction slots 8 g ..;  B: column m, the same slots;  D: column m, rows 4 g .. 4 g + 3).  Codes are
// whole numbers up to 127, exact in bf16, so the scores are products of what is stored, summed in fp32, and the scales come in behind:
// the keys' with the softmax scale, the values' with the probabilities.  Those are split into two bf16 parts, so that they are rounded
// to 16 bits of mantissa (the matrix unit has nothing else to do here).  Row m of key group kg is key 16 (m / 4) + 4 kg + m % 4: lane
// group g then holds the scores of keys 16 g .. 16 g + 15, which are the slots it has to bring as the second product's operand and the
// values it loads as 16 bytes of a row of V^T; nothing is exchanged between lanes but the maximum and the sum.
__device__ __forceinline__ f32x4_t mfma16(bf16x8_t a, bf16x8_t b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// 16 codes that are read once: non-temporal, 131072 keys of 8 heads 52 -> 47 us
typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_once(const void* p) {
    const u32x4_t v = __builtin_nontemporal_load((const u32x4_t*)p);
    return make_uint4(v.x, v.y, v.z, v.w);
}
// eight codes -> bf16
__device__ __forceinline__ bf16x8_t codes_bf16(unsigned lo, unsigned hi) {
    bf16x8_t r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (__bf16)(float)(int8_t)((e < 4 ? lo : hi) >> 8 * (e & 3));
    return r;
}
// eight bf16 of a tail's value row, slots u0 .., zero from slot `end` on; *odd: whether one that stays is not finite
__device__ __forceinline__ uint4 tail_values(uint4 w, int u0, int end, bool* odd) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        unsigned& x = (&w.x)[e];
        if (u0 + 2 * e >= end) x = 0;
        else if (u0 + 2 * e + 1 >= end) x &= 0xffffu;
        *odd |= (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
    }
    return w;
}

// FRESH: the token being decoded, one row of as many query as key heads.  Its q, k and v do not exist as rows yet: every workgroup forms its head's q
// (while its first codes are on their way), and the one whose range ends with the tail forms k and v and puts them there.  The token must not
// complete a block.
// EXACT: complete blocks are held as they came as well, from exact.first on (a kernel of its own: 252 registers instead of 195).
template <int D, int NW, bool FRESH, bool EXACT>
__global__ __launch_bounds__(NW * 64, 8 / NW) void attn8_cols_kernel(Cache8 c, int n_keys, const bf16_t* __restrict__ q, long ldq, int n_rows, int group,
                                                            float scale_log2e, bf16_t* __restrict__ o, long ldo, float* __restrict__ ws,
                                                            int blocks_per_split, DecodeFresh fresh, DecodeOut more, Cache8Exact exact) {
    constexpr int PC = D / 64, NT = D / 16, LDP = D + 4, NCOL = 64 / NW, PART = NCOL * LDP > 1024 ? NCOL * LDP : 1024;
    __shared__ __align__(16) float part[NW][PART];         // a column's output, maximum and sum, wave by wave
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m16 = lane & 15, g = lane >> 4;
    const int head = blockIdx.x, n_cols = n_rows * group, heads = c.heads * group;
    const int col = min(m16, n_cols - 1), row = col / group, seen = n_keys - n_rows + row + 1;      // keys 0 .. seen - 1
    const int least = n_keys - n_rows + 1;                                                              // the first column's
    const int b_begin = (int)blockIdx.y * blocks_per_split, b_end = min(b_begin + blocks_per_split, (n_keys + 63) >> 6);
    const int key0 = (m16 >> 2) * 16 + (m16 & 3), b_tail = n_keys >> 6, b_full = min(b_end, EXACT ? min(b_tail, exact.first) : b_tail);
    // a block's keys are asked for when the block before has used its own, its values when those have been used
    uint4 kr[4][PC], vr[NT];
    float ks_next = 0.f;
    auto keys = [&](int b) {
        const long at = (long)b * c.heads + head;
#pragma unroll
        for (int kg = 0; kg < 4; ++kg)
#pragma unroll
            for (int pc = 0; pc < PC; ++pc) kr[kg][pc] = load_once(c.k + at * 64 * D + pc * 4096 + (key0 + kg * 4) * 64 + g * 16);
        ks_next = c.ks[at];
    };
    int b = b_begin + wave;
    if (b < b_full) keys(b);
    bf16x8_t qf[2 * PC];
    if constexpr (FRESH) {
        constexpr int LPK = D / 8;
        __shared__ float fr[3][D];
        __shared__ __align__(16) bf16_t sq[D];
        __builtin_amdgcn_sched_barrier(0);
        const bool last = b_tail >= b_begin && b_tail < b_end;
        fresh_rows<D, NW * 64>(fresh, head, last, fr);
        const int which = threadIdx.x / LPK, sub = threadIdx.x % LPK, slot = n_keys - 1 & 63;
        __syncthreads();
        if (which == 0 || (which == 1 && last)) {          // q and k, rotated
            float2 cs[8];
            float t[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) cs[e] = fresh.rope[sub % (LPK >> 1) * 8 + e];
            rope8(fr[which] + sub * 8, fr[which] + (sub ^ (LPK >> 1)) * 8, cs, sub, LPK, t);
            bf16_t* to = which ? c.kt + (long)head * 64 * D + (sub >> 3) * 4096 + slot * 64 + (sub & 7) * 8 : sq + sub * 8;
            *(uint4*)to = pack8(t);
        } else if (which == 2 && last) {
#pragma unroll
            for (int e = 0; e < 8; ++e) c.vt[(long)head * 64 * D + (sub * 8 + e) * 64 + slot] = f32_to_bf16(fr[2][sub * 8 + e]);
        }
        __syncthreads();                                   // (the tail's wave reads what the others have stored)
#pragma unroll
        for (int st = 0; st < 2 * PC; ++st) qf[st] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(sq + g * 16 + (st >> 1) * 64 + (st & 1) * 8));
    } else {
        const bf16_t* qr = q + (long)row * ldq + (long)(head * group + col % group) * D + g * 16;
#pragma unroll
        for (int st = 0; st < 2 * PC; ++st) qf[st] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(qr + (st >> 1) * 64 + (st & 1) * 8));
    }

    f32x4_t oacc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) oacc[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    f32x4_t s[4];
    float x[16];
    bf16x8_t hi[2], lo[2];
    // scores -> probabilities (times the values' scale), in two bf16 parts
    auto softmax = [&](int b, float ks, float vs) {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = s[i >> 2][i & 3] * ks;
        if ((b + 1) * 64L > least) {                       // (uniform) some column does not see all of the block
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (b * 64 + g * 16 + i >= seen) x[i] = -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, x[i]);
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float mn = fmaxf(m, top), base = mn == -INFINITY ? 0.f : mn, alpha = __builtin_amdgcn_exp2f(m - base);
        m = mn;
        l *= alpha;
        const float f = (long)b * 64 < seen ? vs : 0.f;    // (a block that a column does not see may have the scale NaN)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[i] = __builtin_amdgcn_exp2f(x[i] - base);
            l += x[i];
            x[i] *= f;
            hi[i >> 3][i & 7] = (__bf16)x[i];
            lo[i >> 3][i & 7] = (__bf16)(x[i] - (float)hi[i >> 3][i & 7]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) oacc[t] *= alpha;
    };
    for (; b < b_full; b += NW) {
        const long at = (long)b * c.heads + head;
#pragma unroll
        for (int t = 0; t < NT; ++t) vr[t] = load_once(c.v + at * 64 * D + (t * 16 + m16) * 64 + g * 16);
        const float ks = ks_next * scale_log2e, vs = c.vs[at];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kg = 0; kg < 4; ++kg) {
            s[kg] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int pc = 0; pc < PC; ++pc) {
                s[kg] = mfma16(codes_bf16(kr[kg][pc].x, kr[kg][pc].y), qf[2 * pc], s[kg]);
                s[kg] = mfma16(codes_bf16(kr[kg][pc].z, kr[kg][pc].w), qf[2 * pc + 1], s[kg]);
            }
            __builtin_amdgcn_sched_barrier(0);             // (widened codes of more than one group would not fit the registers)
        }
        if (b + NW < b_full) keys(b + NW);
        softmax(b, ks, vs);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const bf16x8_t a0 = codes_bf16(vr[t].x, vr[t].y), a1 = codes_bf16(vr[t].z, vr[t].w);
            oacc[t] = mfma16(a0, hi[0], oacc[t]);
            oacc[t] = mfma16(a1, hi[1], oacc[t]);
            oacc[t] = mfma16(a0, lo[0], oacc[t]);
            oacc[t] = mfma16(a1, lo[1], oacc[t]);
            if (t & 1) __builtin_amdgcn_sched_barrier(0);
        }
    }
    for (; b < b_end; b += NW) {                           // the tail, one wave's, and blocks as they came: bf16
        const bool tail = !EXACT || b == b_tail;
        const long at = (tail ? head : (long)(b - exact.first) * c.heads + head) * 64 * D;
        const bf16_t *kt = (tail ? c.kt : exact.k) + at, *vt = (tail ? c.vt : exact.v) + at;
        const int end = tail ? n_keys & 63 : 64;
        bool odd = false;
        uint4 kw[4][2 * PC], vw[NT][2];                    // all of it on its way before the first is used
#pragma unroll
        for (int kg = 0; kg < 4; ++kg)
#pragma unroll
            for (int st = 0; st < 2 * PC; ++st) kw[kg][st] = *(const uint4*)(kt + (st >> 1) * 4096 + (key0 + kg * 4) * 64 + g * 16 + (st & 1) * 8);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) vw[t][h] = *(const uint4*)(vt + (t * 16 + m16) * 64 + g * 16 + h * 8);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kg = 0; kg < 4; ++kg) {
            s[kg] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < 2 * PC; ++st) s[kg] = mfma16(__builtin_bit_cast(bf16x8_t, kw[kg][st]), qf[st], s[kg]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) vw[t][h] = tail_values(vw[t][h], g * 16 + h * 8, end, &odd);
        softmax(b, scale_log2e, 1.f);
        if (!__builtin_amdgcn_ballot_w64(odd)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bf16x8_t a = __builtin_bit_cast(bf16x8_t, vw[t][h]);
                    oacc[t] = mfma16(a, hi[h], oacc[t]);
                    oacc[t] = mfma16(a, lo[h], oacc[t]);
                }
        } else {
            // a value that is not finite counts for the columns that see it alone, which a product with zeros does not give
            float* pl = part[wave];
#pragma unroll
            for (int i = 0; i < 16; ++i) pl[(g * 16 + i) * 16 + m16] = x[i];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            for (int u = 0; u < end && b * 64 + u < seen; ++u) {
                const float p = pl[u * 16 + m16];
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) oacc[t][i] = fmaf(p, bf16_to_f32(vt[(t * 16 + g * 4 + i) * 64 + u]), oacc[t][i]);
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (!EXACT) break;
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (m16 < NCOL) {
        float* mine = part[wave] + m16 * LDP;
#pragma unroll
        for (int t = 0; t < NT; ++t) *(f32x4_t*)(mine + t * 16 + g * 4) = oacc[t];
        if (g == 0) { mine[D] = m; mine[D + 1] = l; }
    }
    uint4 av[4];
    if constexpr (FRESH)
        if (!ws) head_output_fetch<D, NW * 64>(head, heads, more, av);
    __syncthreads();
    float one = 0.f;                                       // FRESH without ranges: this thread's column of the output
    for (int i = threadIdx.x; i < n_cols * D; i += NW * 64) {
        const int cc = i / D, e = i % D;
        float mt = -INFINITY, lt = 0.f, ot = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) mt = fmaxf(mt, part[w][cc * LDP + D]);
        const float base = mt == -INFINITY ? 0.f : mt;     // (of a range that the column sees nothing of)
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float* p = part[w] + cc * LDP;
            const float a = __builtin_amdgcn_exp2f(p[D] - base);
            lt += a * p[D + 1];
            ot += a * p[e];
        }
        const int r = cc / group, qh = head * group + cc % group;
        if (!ws) {
            if constexpr (FRESH) one = ot / lt;
            else o[(long)r * ldo + (long)qh * D + e] = f32_to_bf16(ot / lt);
        } else {
            float* out = ws + (((long)r * heads + qh) * gridDim.y + blockIdx.y) * (D + 2);
            out[e] = ot;
            if (e == 0) { out[D] = mt; out[D + 1] = lt; }
        }
    }
    if constexpr (FRESH)
        if (!ws) head_output<D, NW * 64>(one, threadIdx.x % D, head, heads, more, av);
}

// The ranges of a row and head, one thread a column: lane i holds range i's maximum and sum, and NR ranges' columns are asked for before the first is
// used (6 ranges with NR 8 0.9 us less than with 32).
template <int D, int NR>
__global__ __launch_bounds__(D) void attn8_join_kernel(const float* __restrict__ ws, int n_split, int heads, long ldo, DecodeOut out) {
    const int e = threadIdx.x, lane = threadIdx.x & 63, head = blockIdx.x % heads;
    const float* w = ws + (long)blockIdx.x * n_split * (D + 2);
    const int r = min(lane, n_split - 1);
    const float m = w[r * (D + 2) + D], l = w[r * (D + 2) + D + 1];
    float t[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) t[i] = w[min(i, n_split - 1) * (D + 2) + e];
    uint4 av[8];
    head_output_fetch<D, D>(head, heads, out, av);
    __builtin_amdgcn_sched_barrier(0);
    const float top = wave_max(lane < n_split ? m : -INFINITY);
    const float a = lane < n_split ? __builtin_amdgcn_exp2f(m - top) : 0.f;      // (one range has keys: top is a number, or all is NaN)
    const float sum = wave_sum(lane < n_split ? a * l : 0.f);
    float acc = 0.f;
    for (int i0 = 0; i0 < n_split; i0 += NR) {
        if (i0) {
#pragma unroll
            for (int i = 0; i < NR; ++i) t[i] = w[min(i0 + i, n_split - 1) * (D + 2) + e];
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const float ai = __shfl(a, i0 + i, 64);
            acc += i0 + i < n_split ? ai * t[i] : 0.f;
        }
    }
    out.o += (long)(blockIdx.x / heads) * ldo;
    head_output<D, D>(acc / sum, e, head, heads, out, av);
}

// ---------------------------------------------------------------- attention of many rows
// The same columns, 32 to a wave, NC waves to a workgroup, which takes one tile (a block of the cache) after another:
//   S^T[key][column] = K q^T   and   O^T[d][column] += V^T P^T     by v_mfma_f32_32x32x16_bf16 (operand layout: tiles.h)
// The workgroup's threads widen a tile's codes to bf16 on their way to LDS, each once, so that a code is converted once for 32 NC columns;
// the codes of the tile after are on their way into registers meanwhile, and two buffers make one barrier a tile enough.  Probabilities
// (times the values' scale) are rounded to bf16, as in the attention of a chunk.  16-byte pieces of a row lie in LDS at a place of
// their own for each of 16 rows, so that the fragment reads of 16 lanes meet in no bank; a value row's pieces hold the tokens in the
// order in which a score fragment serves as second operand.
// EXACT: as in the kernel above; those blocks and the tail are tiles of one buffer, loaded when their turn comes (1024 rows and 1024 keys before
// them, 32 heads of 128: 33 us more than over codes; the registers for a tile ahead are not there).
template <int D>
__device__ __forceinline__ unsigned k_piece_at(int key, int c) { return key * D * 2 + ((c ^ (D == 128 ? key & 15 : key >> 1 & 7)) << 4); }
__device__ __forceinline__ unsigned v_piece_at(int d, int c) { return d * 128 + ((c ^ (d >> 1 & 7)) << 4); }

constexpr int ATTN8_ONE_ROUND = 256;                         // workgroups of eight waves that run at once, one a CU

template <int D, int NC, bool EXACT>
__global__ __launch_bounds__(NC * 64, 2) void attn8_rows_kernel(Cache8 c, int n_keys, const bf16_t* __restrict__ q, long ldq, int n_rows, int group,
                                                             float scale_log2e, bf16_t* __restrict__ o, long ldo, float* __restrict__ ws,
                                                             int blocks_per_split, int n_split, Cache8Exact exact) {
    constexpr int KS = D / 16, ND = D / 32, NT = NC * 64, NP = 64 * D / 16, PT = 2 * NP / NT;   // pieces of 16 codes: of K, a thread
    constexpr int TB = 64 * D * 2, STAGE = 2 * TB + 16;                                        // a tile's bytes in LDS, K, V and scales
    extern __shared__ __align__(16) unsigned char smem[];
    int tid = threadIdx.x, l32 = tid & 31, g = tid >> 5 & 1;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // The last columns see most.  Workgroups that all run at once take 128 columns from the end (waves 0 to 3) and as many from the front (4 to 7, on the
    // same SIMDs), so that one has about as much to do as another: 2048 rows of 32 heads and 8192 keys 257 -> 246 us, 2048 keys 63.6 -> 50.9.  Of more, one after
    // another on a CU, those of the last columns come first (4096 rows and keys 146, in pairs 162), as do those of four waves.  A head's workgroups
    // are a multiple of c.heads apart, on one XCD if that is a multiple of eight.
    const bool paired = NC == 8 && gridDim.x <= ATTN8_ONE_ROUND;
    const int n_cols = n_rows * group, heads = c.heads * group, n_parts = (n_cols + 127) / 128, n_blocks = (n_cols + 32 * NC - 1) / (32 * NC);
    const int head = blockIdx.x % c.heads, rest = blockIdx.x / c.heads, split = rest / n_blocks, at = rest % n_blocks;
    const int c0 = (paired ? n_parts - 1 - at : (n_blocks - 1 - at) * (NC / 4)) * 128;         // of waves 0 to 3
    const int w0 = !paired || wave < 4 ? c0 + 32 * wave : 128 * at < c0 ? 128 * at + 32 * (wave - 4) : n_cols;
    const int col = min(w0 + l32, n_cols - 1), row = col / group, seen = n_keys - n_rows + row + 1;
    const int most = n_keys - n_rows + min(c0 + (paired ? 127 : 32 * NC - 1), n_cols - 1) / group + 1;          // keys that the block's last column sees
    const int w_most = w0 < n_cols ? n_keys - n_rows + min(w0 + 31, n_cols - 1) / group + 1 : 0;     // the wave's
    const int w_least = n_keys - n_rows + w0 / group + 1;
    const int b_begin = split * blocks_per_split, b_end = min(b_begin + blocks_per_split, (most + 63) >> 6), b_tail = n_keys >> 6;
    const int b_codes = min(b_end, EXACT ? min(b_tail, exact.first) : b_tail);

    bf16x8_t qf[KS];
    const bf16_t* qr = q + (long)row * ldq + (long)(head * group + col % group) * D + g * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(qr + ks * 16));
    f32x16_t oacc[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) oacc[dt] = zero16();
    float m = -INFINITY, l = 0.f;

    uint4 code[PT];
    float sc = 0.f;                                          // of threads 0 and 1: the tile's scales
    auto fetch = [&](int b) {                                // (of a complete block)
        const long at = (long)b * c.heads + head;
#pragma unroll
        for (int i = 0; i < PT; ++i) {
            const int p = i * NT + tid;
            code[i] = *(const uint4*)((p < NP ? c.k + p * 16 : c.v + (p - NP) * 16) + at * 64 * D);
        }
        if (tid < 2) sc = (tid ? c.vs : c.ks)[at];
    };
    auto widen = [&](unsigned char* st) {
#pragma unroll
        for (int i = 0; i < PT; ++i) {
            const int p = i * NT + tid;
            const uint4 w = code[i];
            if (p < NP) {
                const int key = p >> 2 & 63, ch = (p >> 8) * 8 + (p & 3) * 2;
                *(bf16x8_t*)(st + k_piece_at<D>(key, ch)) = codes_bf16(w.x, w.y);
                *(bf16x8_t*)(st + k_piece_at<D>(key, ch + 1)) = codes_bf16(w.z, w.w);
            } else {
                const int d = (p - NP) >> 2, ch = (p & 3) * 2;
                *(bf16x8_t*)(st + TB + v_piece_at(d, ch)) = codes_bf16(w.x, w.z);
                *(bf16x8_t*)(st + TB + v_piece_at(d, ch + 1)) = codes_bf16(w.y, w.w);
            }
        }
        if (tid < 2) ((float*)(st + 2 * TB))[tid] = tid ? sc : sc * scale_log2e;
    };
    // bf16: the values of the tail, or of a block as it came, and how many tokens of it there are
    auto is_tail = [&](int b) { return !EXACT || b == b_tail; };
    auto exact_at = [&](int b) { return (is_tail(b) ? head : (long)(b - exact.first) * c.heads + head) * 64 * D; };
    auto exact_values = [&](int b) { return (is_tail(b) ? c.vt : exact.v) + exact_at(b); };
    auto exact_tokens = [&](int b) { return is_tail(b) ? n_keys & 63 : 64; };
    // it as a tile; whether a value of it is not finite
    auto exact_tile = [&](int b, unsigned char* st) {
        const bf16_t *kt = (is_tail(b) ? c.kt : exact.k) + exact_at(b), *vt = exact_values(b);
        const int end = exact_tokens(b);
        bool odd = false;
#pragma unroll
        for (int i = 0; i < PT; ++i) {
            const int p = i * NT + tid;
            if (p < NP) {
                const int key = p >> 2 & 63, ch = (p >> 8) * 8 + (p & 3) * 2;
                *(uint4*)(st + k_piece_at<D>(key, ch)) = *(const uint4*)(kt + p * 16);
                *(uint4*)(st + k_piece_at<D>(key, ch + 1)) = *(const uint4*)(kt + p * 16 + 8);
            } else {
                const int d = (p - NP) >> 2, ch = (p & 3) * 2, u0 = (p & 3) * 16;
                const uint4 a = tail_values(*(const uint4*)(vt + d * 64 + u0), u0, end, &odd);
                const uint4 b = tail_values(*(const uint4*)(vt + d * 64 + u0 + 8), u0 + 8, end, &odd);
                *(uint4*)(st + TB + v_piece_at(d, ch)) = make_uint4(a.x, a.y, b.x, b.y);
                *(uint4*)(st + TB + v_piece_at(d, ch + 1)) = make_uint4(a.z, a.w, b.z, b.w);
            }
        }
        if (tid < 2) ((float*)(st + 2 * TB))[tid] = tid ? 1.f : scale_log2e;
        return odd;
    };
    // probs (bf16 [64][32] of this wave) is set for a bf16 tile with values that are not finite
    auto tile = [&](int b, const unsigned char* st, unsigned short* probs) {
        const int u0 = b << 6;
        if (u0 >= w_most) return;                            // (uniform) no column of the wave sees it
        if constexpr (D == 128) __builtin_amdgcn_iglp_opt(0);      // fragment reads between the matrix instructions: 266 -> 257 us; heads of 64 178 -> 181
        f32x16_t s0 = zero16(), s1 = zero16();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            s0 = mfma32(*(const bf16x8_t*)(st + k_piece_at<D>(l32, 2 * ks + g)), qf[ks], s0);
            s1 = mfma32(*(const bf16x8_t*)(st + k_piece_at<D>(32 + l32, 2 * ks + g)), qf[ks], s1);
        }
        // The scales are positive, or NaN: a column that sees nothing of the block takes 1 and 0 instead, so that it learns of no NaN.
        const bool sees = u0 < seen;
        const float ks = sees ? ((const float*)(st + 2 * TB))[0] : 1.f, vs = sees ? ((const float*)(st + 2 * TB))[1] : 0.f;
        if (u0 + 64 > w_least) {                             // some column does not see all of it
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int u = u0 + 8 * (v >> 2) + 4 * g + (v & 3);
                s0[v] = u >= seen ? -INFINITY : s0[v];
                s1[v] = u + 32 >= seen ? -INFINITY : s1[v];
            }
        }
        float x[32], top = s0[0], sum = 0.f;
#pragma unroll
        for (int v = 0; v < 32; ++v) top = fmaxf(top, v < 16 ? s0[v & 15] : s1[v & 15]);
        top = fmaxf(top, __shfl_xor(top, 32, 64)) * ks;
        // m, what the exponents are taken from, follows the maximum only when that is 8 (a factor of 256) ahead: sums and accumulators have the room,
        // and are hardly ever rescaled after the first tiles
        const float mn = top > m + 8.f ? top : m, base = mn == -INFINITY ? 0.f : mn;
        if (__builtin_amdgcn_ballot_w64(mn != m)) {
            const float alpha = __builtin_amdgcn_exp2f(m - base);
            l *= alpha;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int v = 0; v < 16; ++v) oacc[dt][v] *= alpha;
            m = mn;
        }
#pragma unroll
        for (int v = 0; v < 32; ++v) {
            x[v] = __builtin_amdgcn_exp2f(fmaf(v < 16 ? s0[v & 15] : s1[v & 15], ks, -base));
            sum += x[v];
            x[v] *= vs;
        }
        l += sum;
        if (!probs) {
#pragma unroll
            for (int G = 0; G < 4; ++G) {
                const bf16x8_t p = pack_b_from_d(x + 16 * (G >> 1), G & 1);
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
                    oacc[dt] = mfma32(*(const bf16x8_t*)(st + TB + v_piece_at(dt * 32 + l32, 2 * G + g)), p, oacc[dt]);
            }
        } else {
            // a value that is not finite counts for the columns that see it alone, which a product with zeros does not give
            const bf16_t* vt = exact_values(b);
#pragma unroll
            for (int v = 0; v < 32; ++v) probs[(32 * (v >> 4) + 8 * (v >> 2 & 3) + 4 * g + (v & 3)) * 32 + l32] = f32_to_bf16(x[v]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            for (int u = 0; u < exact_tokens(b) && u0 + u < seen; ++u) {
                const float p = bf16_to_f32(probs[u * 32 + l32]);
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                    for (int v = 0; v < 16; ++v) oacc[dt][v] = fmaf(p, bf16_to_f32(vt[(dt * 32 + 8 * (v >> 2) + 4 * g + (v & 3)) * 64 + u]), oacc[dt][v]);
            }
        }
    };

    const int full = b_codes - b_begin;                      // blocks that are codes
    if (full > 0) {
        fetch(b_begin);
        widen(smem);
        if (full > 1) fetch(b_begin + 1);
    }
    for (int i = 0; i < full; ++i) {
        __syncthreads();                                     // tile i is there, tile i - 1 has been read
        if (i + 1 < full) widen(smem + (i + 1 & 1) * STAGE);
        if (i + 2 < full) fetch(b_begin + i + 2);
        tile(b_begin + i, smem + (i & 1) * STAGE, nullptr);
    }
    for (int b = max(b_begin, b_codes); b < b_end; ++b) {    // blocks as they came, and the tail
        // (opaque: the places in LDS are worked out tile by tile, or they would be kept beside all else and 130 bytes a lane spilled)
        if constexpr (EXACT) asm volatile("" : "+v"(tid), "+v"(l32), "+v"(g));
        __syncthreads();
        const bool odd = exact_tile(b, smem);
        unsigned short* probs = (unsigned short*)(smem + STAGE) + wave * 64 * 32;
        if (__syncthreads_or(odd)) tile(b, smem, probs);
        else tile(b, smem, nullptr);
        if (!EXACT) break;
    }
    l += __shfl_xor(l, 32, 64);
    if (n_split > 1) {
        if (w0 + l32 >= n_cols) return;
        float* out = ws + (((long)row * heads + head * group + col % group) * n_split + split) * (D + 2);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int v = 0; v < 16; v += 2) *(float2*)(out + dt * 32 + 8 * (v >> 2) + 4 * g + (v & 3)) = make_float2(oacc[dt][v], oacc[dt][v + 1]);
        if (g == 0) *(float2*)(out + D) = make_float2(m, l);
        return;
    }
    __syncthreads();
    constexpr int LD = D + 8;
    bf16_t* slab = (bf16_t*)smem + wave * 32 * LD;           // the wave's 32 columns leave in 16-byte pieces
    const float inv = 1.f / l;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int v = 0; v < 16; v += 4)
            *(uint2*)(slab + l32 * LD + dt * 32 + 2 * v + 4 * g) = make_uint2(pack_bf16x2(oacc[dt][v] * inv, oacc[dt][v + 1] * inv),
                                                                            pack_bf16x2(oacc[dt][v + 2] * inv, oacc[dt][v + 3] * inv));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = lane; i < 32 * D / 8; i += 64) {
        const int cc = w0 + i / (D / 8), e = i % (D / 8) * 8;
        if (cc < n_cols) *(uint4*)(o + (long)(cc / group) * ldo + (long)(head * group + cc % group) * D + e) = *(const uint4*)(slab + (i / (D / 8)) * LD + e);
    }
}
// two tiles; the probabilities behind the first of them; the output slab
template <int D, int NC>
static constexpr size_t attn8_rows_lds() {
    constexpr size_t stage = 2 * 64 * D * 2 + 16;
    return std::max({2 * stage, stage + NC * 64 * 32 * 2, (size_t)NC * 32 * (D + 8) * 2});
}

// Which kernel, and how the keys are cut.
//   columns16, columns8  up to 16 columns of a key head: four waves for 16 columns, or eight for 8 that share the blocks of a range.  us for 2 rows of 32
//                     heads of 128, this and rows128: 300 keys 8.2 and 8.1, 1500 9.5 and 12.5, 4000 12.2 and 18.6; 17 rows: 300 keys 10.2 and 8.7,
//                     1500 13.3 and 13.2, 4000 19.1 and 15.5
//   rows128, rows256  more columns, 128 or 256 to a workgroup (both, 32 heads: 2048 rows of 8 key heads, 8192 keys 277 and 246; 1024 rows, 2048 keys 52 and 57; 200 rows,
//                     4000 keys in 8 ranges 37.2 and 34.5; 200 rows of 4 heads in 16 16.7 and 19.0)
// Ranges of few columns: none up to 11 blocks, from 5 on with eight waves (one row of 32 heads, 500 keys: 7.8 with four waves, 7.5 with eight, 8.0 cut; 700
// keys 10.1, 8.4, 8.2 and a launch more; 1000 keys 12.4, 11.9, 8.3).  Else two workgroups a CU, of three blocks or more, but one a CU where each has over
// 16 blocks (32768 keys of 32 heads 50.9 and 48.2).  Where that is over 16 ranges (few key heads), 16 of up to four blocks
// (4000 keys of 8 heads: 16 8.9, 21 9.9) or 32 of eight waves (16000 keys of 8 heads: 64 of four
// waves 14.4, 32 of eight 12.3), from 512 blocks on as many as leave a workgroup for each CU (65536 keys of 2 heads: 32 21.8, 64 16.4; 8000 keys of one: 32
// 9.1, 42 10.3).
// Many columns: the workgroup and the ranges that cost least of a launch's tiles one after another (1.75 us each with one workgroup of 128 columns on a
// CU, 2.7 with two; 2.3 of 256 columns, 1.75 where half of them does not see the tile) and of the join (3 us, and its floats written and read at 3.5 TB/s).
struct Attn8Plan { int cols, waves, n_split, per; };       // columns and waves a workgroup, ranges, blocks a range
static Attn8Plan attn8_plan(int n_keys, int n_rows, int heads, int kv_heads, int d, size_t ws_elems) {
    const int nb = cdiv(n_keys, 64);
    const long n_cols = (long)n_rows * (heads / kv_heads);
    const long range_elems = (long)n_rows * heads * (d + 2);
    const long most = std::min<long>(std::min<long>(nb, ATTN8_MAX_SPLIT), (long)(ws_elems / (size_t)range_elems));
    long n = 1;
    int cols = 16, waves = 4;
    if (n_cols <= 16) {
        const long units = kv_heads;
        if (nb > 11) {
            n = std::min<long>(512 / units, cdiv(nb, 3));
            if (n > 16 && nb <= 64) n = 16;
            else if (n > 16 && n_cols <= 8) {
                waves = 8;
                n = std::min(n, nb > 512 ? std::max(32l, 256 / units) : 32l);
            } else if (n > 1 && cdiv(nb, n) > 16) n = 256 / units;
        }
        n = std::min(n, most);
        if (n < 2 && nb > 4 && n_cols <= 8) waves = 8;
    } else {
        double best = 0.;
        for (int c : {128, 256}) {
            if (c > 128 && n_cols <= 128) break;
            const long units = kv_heads * (long)cdiv(n_cols, c), slots = c == 128 ? 2 * ATTN8_ONE_ROUND : ATTN8_ONE_ROUND;
            for (long r = 1; r == 1 || r <= most; ++r) {
                const long w = units * r, rest = w % slots;
                const double tile = c == 128 ? 2.7 : 2.3, last = rest == 0 ? 0. : c == 128 && rest <= ATTN8_ONE_ROUND ? 1.75 : tile;
                double cost = cdiv(nb, r) * ((double)(w / slots) * tile + last) + (r > 1 ? 3. + 8. * r * range_elems / 3.5e6 : 0.);
                if (c > 128 && w <= ATTN8_ONE_ROUND && r == 1) cost -= (2.3 - 1.75) * (n_rows / 64);      // (in pairs: half of the waves has as many fewer)
                if ((c == 128 && r == 1) || cost < best) best = cost, cols = c, n = r;
            }
        }
        waves = cols / 32;
    }
    if (n < 2) return {cols, waves, 1, nb};
    const int per = cdiv(nb, n);
    return {cols, waves, cdiv(nb, per), per};
}
const char* attention_cache8_plan(int n_keys, int n_rows, int heads, int kv_heads, int d, size_t ws_elems, int* n_ranges) {
    const Attn8Plan p = attn8_plan(n_keys, n_rows, heads, kv_heads, d, ws_elems);
    *n_ranges = p.n_split;
    return p.cols == 16 ? (p.waves == 8 ? "columns8" : "columns16") : p.cols == 128 ? "rows128" : "rows256";
}
template <int D>
static hipError_t run_attention_cache8(const Attn8Plan& p, const Cache8& c, int n_keys, const bf16_t* q, long ldq, int n_rows, int group, bf16_t* o,
                                       long ldo, float* ws, hipStream_t s, const DecodeFresh* fresh, const DecodeOut& out,
                                       const Cache8Exact& exact = Cache8Exact{}) {
    const float scale = 1.4426950408889634f / sqrtf((float)D);
    const long n_cols = (long)n_rows * group;
    float* w = p.n_split > 1 || (out.a && !fresh) ? ws : nullptr;       // (the join leaves the shares of A o)
    auto rows = [&](auto nc, auto kernel) {
        constexpr int NC = decltype(nc)::value;
        constexpr size_t lds = attn8_rows_lds<D, NC>();
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
        kernel<<<c.heads * cdiv(n_cols, 32 * NC) * p.n_split, NC * 64, lds, s>>>(c, n_keys, q, ldq, n_rows, group, scale, o, ldo, w,
                                                                                             p.per, p.n_split, exact);
        return hipGetLastError();
    };
    hipError_t e;
    if (p.cols == 16) {                                    // (one workgroup holds all the columns of a key head)
        auto cols = [&](auto kernel, int threads) {
            kernel<<<dim3(c.heads, p.n_split), threads, 0, s>>>(c, n_keys, q, ldq, n_rows, group, scale, o, ldo, w, p.per, fresh ? *fresh : DecodeFresh{}, out,
                                                               exact);
        };
        if (fresh) p.waves == 8 ? cols(attn8_cols_kernel<D, 8, true, false>, 512) : cols(attn8_cols_kernel<D, 4, true, false>, 256);
        else if (exact.k) p.waves == 8 ? cols(attn8_cols_kernel<D, 8, false, true>, 512) : cols(attn8_cols_kernel<D, 4, false, true>, 256);
        else p.waves == 8 ? cols(attn8_cols_kernel<D, 8, false, false>, 512) : cols(attn8_cols_kernel<D, 4, false, false>, 256);
        e = hipGetLastError();
    } else if (p.cols == 128) {
        constexpr std::integral_constant<int, 4> nc;
        e = exact.k ? rows(nc, attn8_rows_kernel<D, 4, true>) : rows(nc, attn8_rows_kernel<D, 4, false>);
    } else {
        constexpr std::integral_constant<int, 8> nc;
        e = exact.k ? rows(nc, attn8_rows_kernel<D, 8, true>) : rows(nc, attn8_rows_kernel<D, 8, false>);
    }
    if (e != hipSuccess || !w) return e;
    auto join = p.n_split <= 8 ? attn8_join_kernel<D, 8> : p.n_split <= 16 ? attn8_join_kernel<D, 16> : attn8_join_kernel<D, 32>;
    join<<<n_rows * c.heads * group, D, 0, s>>>(w, p.n_split, c.heads * group, ldo, out);
    return hipGetLastError();
}
hipError_t launch_attention_cache8(const Cache8& c, int n_keys, const bf16_t* q, long ldq, int n_rows, int heads, bf16_t* o, long ldo,
                                   float* ws, size_t ws_elems, hipStream_t s, const Cache8Exact& exact) {
    if (n_rows <= 0) return n_rows == 0 ? hipSuccess : hipErrorInvalidValue;
    const Attn8Plan p = attn8_plan(n_keys, n_rows, heads, c.heads, c.d, ws ? ws_elems : 0);
    DecodeOut out;
    out.o = o;
    return c.d == 128 ? run_attention_cache8<128>(p, c, n_keys, q, ldq, n_rows, heads / c.heads, o, ldo, ws, s, nullptr, out, exact)
                      : run_attention_cache8<64>(p, c, n_keys, q, ldq, n_rows, heads / c.heads, o, ldo, ws, s, nullptr, out, exact);
}

// ---------------------------------------------------------------- the token being decoded
// The rows q | k | v of a token, [3 d] bf16, q and k rotated: one workgroup a head.
template <int D>
__global__ __launch_bounds__(256) void decode_token_kernel(DecodeFresh fresh, bf16_t* __restrict__ qkv) {
    constexpr int LPK = D / 8;
    __shared__ float fr[3][D];
    const int head = blockIdx.x, which = threadIdx.x / LPK, sub = threadIdx.x % LPK;
    fresh_rows<D, 256>(fresh, head, true, fr);
    __syncthreads();
    if (which > 2) return;
    float t[8];
    if (which < 2) {
        float2 cs[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) cs[e] = fresh.rope[sub % (LPK >> 1) * 8 + e];
        rope8(fr[which] + sub * 8, fr[which] + (sub ^ (LPK >> 1)) * 8, cs, sub, LPK, t);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = fr[2][sub * 8 + e];
    }
    *(uint4*)(qkv + (long)which * fresh.d + (long)head * D + sub * 8) = pack8(t);
}
// Puts the token into the cache as token n_keys - 1 and attends to all n_keys: in the attention launch itself, but for one token in 64, which completes
// a block: its rows are formed, appended (the block becomes codes) and attended with one after another, in `qkv` ([3 d], scratch).
hipError_t launch_decode_cache8(const Cache8& c, int n_keys, const DecodeFresh& fresh, const DecodeOut& out, bf16_t* qkv, float* ws, size_t ws_elems,
                                hipStream_t s) {
    if (n_keys < 1 || fresh.d != c.heads * c.d || (fresh.r & 7) || (out.a && (out.r & 7)) || !ws || ws_elems < (size_t)fresh.d + 2 * c.heads) return hipErrorInvalidValue;
    const Attn8Plan p = attn8_plan(n_keys, 1, c.heads, c.heads, c.d, ws ? ws_elems : 0);
    const bool whole = (n_keys & 63) == 0;
    if (whole) {
        if (c.d == 128) decode_token_kernel<128><<<c.heads, 256, 0, s>>>(fresh, qkv);
        else decode_token_kernel<64><<<c.heads, 256, 0, s>>>(fresh, qkv);
        hipError_t e = hipGetLastError();
        if (e == hipSuccess) e = launch_cache8_append(c, n_keys - 1, qkv + fresh.d, 3L * fresh.d, qkv + 2L * fresh.d, 3L * fresh.d, 1, s);
        if (e != hipSuccess) return e;
    }
    return c.d == 128 ? run_attention_cache8<128>(p, c, n_keys, qkv, 3L * fresh.d, 1, 1, out.o, fresh.d, ws, s, whole ? nullptr : &fresh, out)
                      : run_attention_cache8<64>(p, c, n_keys, qkv, 3L * fresh.d, 1, 1, out.o, fresh.d, ws, s, whole ? nullptr : &fresh, out);
}
