// A token drawn from each row of logits: temperature, top-k, top-p, min-p, and a given number.
//   w_i = round(2^40 exp((x_i - largest) / temperature))      whole numbers, so that sums of them are exact in any order
// The order is that of the logits, the lowest index first among equals.  Kept are the first top_k of it, of these the ones that less than top_p of
// their weight lies before, of these the ones with at least min_p of the largest weight.  With S the kept weight, the token is the first in the order
// of the indices up to which more than floor(u S) is kept.
#include <type_traits>

#include "kernels.h"

typedef unsigned long long u64;
constexpr u64 SAMPLE_ONE = 1ull << 40;
constexpr int SAMPLE_BINS = 2048;
constexpr float SAMPLE_REACH = 1846.f;     // 64 units of the bins to one of (largest - x) / temperature: what lies further than 28.84 weighs less than half a unit

// p f + c with a constant of all lanes (the compiler takes the form that adds to its third operand, and copies the constant there before each)
__device__ __forceinline__ double fma_by(double p, double f, double c) {
    double r;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(p), "v"(f), "s"(c));
    return r;
}
// 2^y in units of 2^-40, y <= 0 (NaN: 0), rounded to the nearest: 2^n 2^f with y = n + f, |f| <= 1/2, 2^f by the polynomial of the 10th degree that equals it at the
// 11 Chebyshev points of [-1/2, 1/2] (solved for in 50 digits; with its coefficients in fp64 it is off by 2^-51.5 of 2^f at most, as several of an fp64 sum's
// roundings are).  n goes into the exponent; adding 2^52 rounds to a whole number and leaves it in the mantissa's low bits.
__device__ __forceinline__ u64 weight_of(double y) {
    y = fmax(y, -60.0);
    const double n = rint(y), f = y - n;
    double p = 7.072585949269223e-09;
    p = fma_by(p, f, 1.0208690299958306e-07);
    p = fma_by(p, f, 1.321544258792169e-06);
    p = fma_by(p, f, 1.5252657260200837e-05);
    p = fma_by(p, f, 0.0001540353044173605);
    p = fma_by(p, f, 0.0013333558230164974);
    p = fma_by(p, f, 0.009618129107606888);
    p = fma_by(p, f, 0.05550410866444772);
    p = fma_by(p, f, 0.24022650695910097);
    p = fma_by(p, f, 0.69314718055995);
    p = fma(p, f, 1.0);
    p = __hiloint2double(__double2hiint(p) + (((int)n + 40) << 20), __double2loint(p)) + 4503599627370496.0;
    return (u64)__double_as_longlong(p) & 0xfffffffffffffull;
}
// larger for larger x, the same for 0 and -0
__device__ __forceinline__ unsigned key_of_logit(float x) {
    const unsigned u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of_key(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
// a place in the order, larger: earlier
__device__ __forceinline__ u64 composite(float v, int i) { return (u64)key_of_logit(v) << 22 | (unsigned)(0x3fffff - i); }
__device__ __forceinline__ float logit_of(u64 e) { return logit_of_key((unsigned)(e >> 22)); }
__device__ __forceinline__ int index_of(u64 e) { return 0x3fffff - (int)(e & 0x3fffff); }

// a value of another lane of the wave by DPP (lanes without one: 0); 64 bits as two halves
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ u64 dpp(u64 v) {
    return (u64)(unsigned)dpp<CTRL, ROWS>((int)(v >> 32)) << 32 | (unsigned)dpp<CTRL, ROWS>((int)(unsigned)v);
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float dpp(float v) { return __int_as_float(dpp<CTRL, ROWS>(__float_as_int(v))); }
// inclusive sums over the lanes of a wave: along rows of 16, then the rows' ends into the rows behind
template <class N>
__device__ __forceinline__ N wave_scan(N v) {
    v += dpp<0x111>(v);                                    // row_shr:1
    v += dpp<0x112>(v);
    v += dpp<0x114>(v);
    v += dpp<0x118>(v);
    v += dpp<0x142, 0xa>(v);                               // row_bcast:15 into rows 1 and 3
    v += dpp<0x143, 0xc>(v);                               // row_bcast:31 into rows 2 and 3
    return v;
}
// the value of lane ^ j
__device__ __forceinline__ u64 lane_xor(u64 v, int j) {
    switch (j) {
        case 1: return dpp<0xb1>(v);                       // quad_perm
        case 2: return dpp<0x4e>(v);
        case 4: return dpp<0x1b>(dpp<0x141>(v));           // mirrored in half rows, mirrored in fours
        case 8: return dpp<0x128>(v);                      // row_ror:8
        default: return __shfl_xor(v, j, 64);
    }
}

template <int NT, int LIST>
struct SampleLds {
    u64 sum[SAMPLE_BINS];
    int count[SAMPLE_BINS];
    u64 list[LIST];
    u64 wave_sum[NT / 64];
    u64 found_sum, found_before_sum, lowest;
    int found, found_count, found_before, n_list;
    float about;
};
// inclusive sums over the threads of the workgroup; the total to *all
template <class S, class N>
__device__ __forceinline__ N block_scan(S& s, N v, N* all) {
    constexpr int NW = sizeof(s.wave_sum) / sizeof(u64);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    v = wave_scan(v);
    N* ends = (N*)s.wave_sum;
    __syncthreads();
    if (lane == 63) ends[wave] = v;
    __syncthreads();
    N total = 0;
#pragma unroll 4
    for (int w = 0; w < NW; ++w) {
        const N o = ends[w];
        if (w < wave) v += o;
        total += o;
    }
    *all = total;
    return v;
}
// the bin in which the count (by_count) or the weight, summed up from bin 0 and on top of before_*, first reaches `limit`: s.found (-1: none does), its own
// count and sum, and those before it.  SUMS: else the counts alone are there and wanted.
template <int NT, bool SUMS, class S>
__device__ __forceinline__ void find_bin(S& s, bool by_count, u64 limit, int before_count, u64 before_sum) {
    constexpr int N = SAMPLE_BINS / NT;
    const int b = N * threadIdx.x;
    int c[N], cs = 0;
    u64 w[N], ws = 0, all;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        c[i] = s.count[b + i], cs += c[i];
        w[i] = SUMS ? s.sum[b + i] : 0, ws += w[i];
    }
    if (threadIdx.x == 0) s.found = -1;
    int all_c;
    cs = block_scan(s, cs, &all_c) - cs + before_count;
    if (SUMS) ws = block_scan(s, ws, &all) - ws + before_sum;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const u64 start = by_count ? (u64)cs : ws, end = by_count ? (u64)(cs + c[i]) : ws + w[i];
        if (start < limit && limit <= end) s.found = b + i, s.found_count = c[i], s.found_sum = w[i], s.found_before = cs, s.found_before_sum = ws;
        cs += c[i], ws += w[i];
    }
    __syncthreads();
}
// The same where about so much weighs: in the place of the counts lie the tokens' weights as parts of the largest that the bin has room for, whole
// numbers in units of 2^-bits.  (32-bit sums of whole numbers are several times faster here than of 64 bits, or of floating point.)  Where the place lies next to a
// border, s.found and *last are the bins on both sides: a row whose cut lies beside the bin found is read twice more (before, one of some thousands: a call of 256 rows 145
// instead of 89 us).  Returns what weighs up to the last one's end, in units of the largest weight.
template <int NT, class S>
__device__ __forceinline__ float find_about(S& s, float p, int bits, int* last) {
    constexpr int N = SAMPLE_BINS / NT;
    const int b = N * threadIdx.x;
    float w[N], ws = 0.f, all;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = (float)(unsigned)s.count[b + i] * __builtin_amdgcn_exp2f((float)(b + i) * (-1.44269504088896340736f / 64.f) - (float)bits), ws += w[i];
    if (threadIdx.x == 0) s.found = SAMPLE_BINS - 1, s.found_count = 0, s.about = 0.f;       // (nowhere: roundings, and the caller finds out)
    const float mine = ws;
    ws = block_scan(s, ws, &all) - mine;
    const float slack = all * __builtin_amdgcn_exp2f((float)(-bits - 4)), low = p * all - slack, high = p * all + slack;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float end = ws + w[i];
        if (w[i] > 0.f && (ws < high || b + i == 0) && low <= end) {
            atomicMin(&s.found, b + i);
            atomicMax(&s.found_count, b + i);
            atomicMax((int*)&s.about, __float_as_int(end));        // (both above 0)
        }
        ws = end;
    }
    __syncthreads();
    *last = max(s.found, s.found_count);
    return s.about;
}
// one value a thread, the largest in thread 0; n of them are not 0
template <class S>
__device__ __forceinline__ u64 block_sort(S& s, u64 v, int n) {
    int size = 64;
    while (size < n) size <<= 1;
    const int t = threadIdx.x;
    auto keep = [&](u64 o, int k, int j) {
        const bool larger = ((t & k) == 0) == ((t & j) == 0);          // this one keeps the larger
        v = larger == (v > o) ? v : o;
    };
    auto in_wave = [&](int k) {
        if (k >= 64) keep(lane_xor(v, 32), k, 32);
        if (k >= 32) keep(lane_xor(v, 16), k, 16);
        if (k >= 16) keep(lane_xor(v, 8), k, 8);
        if (k >= 8) keep(lane_xor(v, 4), k, 4);
        if (k >= 4) keep(lane_xor(v, 2), k, 2);
        keep(lane_xor(v, 1), k, 1);
    };
#pragma unroll
    for (int k = 2; k <= 64; k <<= 1) in_wave(k);
    for (int k = 128; k <= size; k <<= 1) {
        for (int j = k >> 1; j >= 64; j >>= 1) {
            __syncthreads();
            s.list[t] = v;
            __syncthreads();
            keep(s.list[t ^ j], k, j);
        }
        in_wave(k);
    }
    return v;
}

// What a row's pieces have found out before its one workgroup draws from it (few rows of many tokens, see launch_sample)
constexpr int SAMPLE_PIECE = 8192, SAMPLE_CHUNK = 512;
struct SampleFound {
    u64* best;                            // [rows][pieces] a piece's largest as composite (0: none)
    u64* sum;                             // [rows][SAMPLE_BINS] the bins' weights, or, without top_k and top_p, what is kept of each SAMPLE_CHUNK tokens
    int* count;                           // [rows][SAMPLE_BINS + 1] the bins' tokens (with top_k; their weights without); how many tokens are kept
    int pieces;
};
// how the tokens of a row are weighed
struct SampleRow {
    float half, to_bins;                  // half the largest; bins to half a unit of a logit (halves: a difference of two logits may overflow)
    double top64, per;                    // per: log2(e) / temperature
    __device__ __forceinline__ SampleRow(float top, float temperature)
        : half(0.5f * top), to_bins(fminf(128.f / temperature, 3e38f)), top64((double)top), per(1.0 / (double)temperature * 1.44269504088896340736) {}
    __device__ __forceinline__ u64 weight(float v) const { return weight_of(((double)v - top64) * per); }
    __device__ __forceinline__ float place_below(float from, float v) const { return fmaf(-0.5f, v, from) * to_bins; }
    __device__ __forceinline__ float place(float v) const { return place_below(half, v); }      // monotone, as each step of it is; its whole part is the bin
};
__device__ __forceinline__ u64 least_weight(float min_p) {
    return !(min_p > 0.f) ? 1ull : min_p >= 1.f ? SAMPLE_ONE : (u64)ceil((double)min_p * (double)SAMPLE_ONE);
}
// How far below the largest, in temperatures, a weight that rounds to `least` lies at most, and a little more for the roundings of what is compared with it
__device__ __forceinline__ float reach_of_least(u64 least) { return 0.001f - __logf(((float)least - 0.5f) * 0x1p-40f); }
__device__ __forceinline__ int wanted(float top_k, int vocab) { return top_k >= 1.f && top_k < (float)vocab ? (int)top_k : 0; }
// the larger of all lanes' composites, in every lane
__device__ __forceinline__ u64 wave_best(u64 v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const u64 o = __shfl_xor(v, off, 64);
        v = v > o ? v : o;
    }
    return v;
}
__device__ __forceinline__ u64 row_best(const SampleFound& w, long r, int lane) {
    u64 best = 0;
    for (int i = lane; i < w.pieces; i += 64) best = best > w.best[r * w.pieces + i] ? best : w.best[r * w.pieces + i];
    return wave_best(best);
}
// eight tokens of a piece a thread, one chunk a wave: 64 lanes x 4, twice
template <class F>
__device__ __forceinline__ void each_of_piece(const float* x, int vocab, F&& f) {
    const int i0 = (int)blockIdx.x * SAMPLE_PIECE + (threadIdx.x >> 6) * SAMPLE_CHUNK + (threadIdx.x & 63) * 4;
    float4 v[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = i0 + k * 256;
        if (i + 4 <= vocab) v[k] = *(const float4*)(x + i);
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e) (&v[k].x)[e] = i + e < vocab ? x[i + e] : -INFINITY;
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) f((&v[k].x)[e], i0 + k * 256 + e);
}
__global__ __launch_bounds__(1024) void sample_best_kernel(Sample c, int vocab, SampleFound w) {
    __shared__ u64 part[16];
    const long r = blockIdx.y;
    u64 best = 0;
    each_of_piece(c.logits + r * c.ldl, vocab, [&](float v, int i) {
        const u64 e = v > -INFINITY ? composite(v, i) : 0;
        best = best > e ? best : e;
    });
    best = wave_best(best);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = best;
    for (int i = blockIdx.x * 1024 + threadIdx.x; i < SAMPLE_BINS; i += gridDim.x * 1024) w.sum[r * SAMPLE_BINS + i] = 0, w.count[r * (SAMPLE_BINS + 1) + i] = 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) w.count[r * (SAMPLE_BINS + 1) + SAMPLE_BINS] = 0;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 16; ++i) best = best > part[i] ? best : part[i];
        w.best[r * w.pieces + blockIdx.x] = best;
    }
}
__global__ __launch_bounds__(1024) void sample_weigh_kernel(Sample c, int vocab, SampleFound w) {
    __shared__ u64 sum[SAMPLE_BINS];
    __shared__ int count[SAMPLE_BINS];
    const long r = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 63;
    const float* params = c.params ? c.params + r * c.ldp : c.now;
    const float temperature = params[0], top_k = params[1], top_p = params[2], min_p = params[3];
    float top = logit_of(row_best(w, r, lane));
    if (!(temperature > 0.f) || !(top > -INFINITY)) return;
    const bool infinite = top == INFINITY;
    const SampleRow row(infinite ? 0.f : top, temperature);
    auto each = [&](auto&& f) { each_of_piece(c.logits + r * c.ldl, vocab, [&](float v, int) { f(!infinite ? v : v == INFINITY ? 0.f : -INFINITY); }); };
    const bool by_count = wanted(top_k, vocab) > 0;        // (the weights are not looked at then, or weighed again)
    if (by_count || top_p < 1.f) {
        for (int i = tid; i < SAMPLE_BINS; i += 1024) sum[i] = 0, count[i] = 0;
        __syncthreads();
        each([&](float v) {
            const float b = row.place(v);
            if (!(b < SAMPLE_REACH)) return;
            if (by_count) atomicAdd(&count[(int)b], 1);
            else atomicAdd(&sum[(int)b], row.weight(v));
        });
        __syncthreads();
        for (int i = tid; i < SAMPLE_BINS; i += 1024) {
            if (count[i]) atomicAdd(w.count + r * (SAMPLE_BINS + 1) + i, count[i]);
            if (sum[i]) atomicAdd(w.sum + r * SAMPLE_BINS + i, sum[i]);
        }
    } else {
        const u64 least = least_weight(min_p);
        u64 all = 0;
        int n = 0;
        each([&](float v) {
            const u64 x = row.weight(v);
            if (x >= least) all += x, ++n;
        });
        all = wave_scan(all);
        n = wave_scan(n);
        if (lane == 63) {
            const int at = (int)blockIdx.x * (SAMPLE_PIECE / SAMPLE_CHUNK) + (tid >> 6);
            if (at < SAMPLE_BINS) w.sum[r * SAMPLE_BINS + at] = all;
            if (n) atomicAdd(w.count + r * (SAMPLE_BINS + 1) + SAMPLE_BINS, n);
        }
    }
}

// One workgroup a row.  HELD: the row stays in LDS from its one reading on; else every pass over it reads it again.
//   pass 1  the largest logit
//   pass 2  with top_k: the tokens in each of 2048 ranges of (largest - x) / temperature, 64 to a unit, are counted (few wanted: the range that the threads' own
//           largest say is enough, without counting); with top_p: about how much lies in each
//   pass 3  what lies in the ranges up to the one with the cut is listed; up to a token a thread, the list is sorted, cut and drawn from.  With top_p this pass
//           weighs all tokens, each exactly and once; if more are kept than the list holds, it sums up what lies before the range and lists the range alone
//   else    the cut is found digit by digit among the tokens of its range (from a list if they fit one), and a last pass draws
// Where a row has to be read again, passes 1 and 2 are one, from what the first logits say of the largest (anchored), or all three are (listed).
// FOUND: passes 1 and 2, and without top_k and top_p the last one's sums, have been made by the row's pieces.
// What bounds it: a weight is 21 instructions of the vector unit, most in fp64 (35 us for all tokens of 512 rows of 128000), and with what goes on around it 25 to 50;
// reading those once is 47 us (5.6 TB/s, the greedy call), and what does not fit a CU is read two or three times.  512 rows of 128000: without a limit 110 us, min-p 59,
// top-k 50 59, top-k 400 93 (124 with a pass of its own to count), top-k 1000 217, top-p 0.9 148 to 156, greedy 47.  One row of 32000, in LDS: 15, 11, 13, 22, 24 and 8 (a call that does nothing: 6); what bounds it is the chain of
// barriers, scans and sorts on one CU.
template <int NT, int LIST, bool HELD, bool FOUND>
__global__ __launch_bounds__(NT, 4) void sample_kernel(Sample c, int vocab, SampleFound found_in) {
    constexpr int NW = NT / 64;
    __shared__ SampleLds<NT, LIST> s;
    extern __shared__ __align__(16) float held[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long r = blockIdx.x;
    const float* x = c.logits + r * c.ldl;
    const float* params = c.params ? c.params + r * c.ldp : c.now;
    const float temperature = params[0], top_k = params[1], top_p = params[2], min_p = params[3], u = c.u ? c.u[r] : c.now_u;
    auto out = [&](int choice, int kept, float prob) {
        c.choice[r] = choice;
        if (c.kept) c.kept[r] = kept;
        if (c.prob) c.prob[r] = prob;
    };
    bool infinite = false;                                 // the largest is infinity: its equals count as 0, all others as -infinity
    auto from_memory = [&](int i) __attribute__((always_inline)) -> float4 {              // (behind the row: -infinity, which weighs nothing)
        float4 v;
        if (i + 4 <= vocab) v = *(const float4*)(x + i);
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e) (&v.x)[e] = i + e < vocab ? x[i + e] : -INFINITY;
        }
        return v;
    };
    // f(x[i], i), the lanes side by side, from the first on to the end, both multiples of 4; U times four a lane at a time, the next on their way
    auto each = [&](auto lanes, int first, int end, int at, auto&& f) __attribute__((always_inline)) {
        constexpr int LANES = decltype(lanes)::value, U = HELD ? 1 : FOUND ? 2 : 4;
        float4 v[U], next[U];
        auto fetch = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int i = i0 + (k * LANES + at) * 4;
                if (i >= end) next[k] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                else if (HELD) next[k] = *(const float4*)(held + i);
                else next[k] = from_memory(i);
            }
        };
        fetch(first);
        for (int i0 = first; i0 < end; i0 += 4 * LANES * U) {
#pragma unroll
            for (int k = 0; k < U; ++k) v[k] = next[k];
            fetch(i0 + 4 * LANES * U);
            if (!HELD && infinite) {
#pragma unroll
                for (int k = 0; k < U; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) (&v[k].x)[e] = (&v[k].x)[e] == INFINITY ? 0.f : -INFINITY;
            }
#pragma unroll
            for (int k = 0; k < U; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f((&v[k].x)[e], i0 + (k * LANES + at) * 4 + e);
                    if (e & 1) __builtin_amdgcn_sched_barrier(0);        // (more than two weights at a time would not fit the registers)
                }
        }
    };
    const int padded = (vocab + 3) & ~3;
    auto all_of = [&](auto&& f) __attribute__((always_inline)) { each(std::integral_constant<int, NT>{}, 0, padded, tid, f); };

    const bool greedy = !(temperature > 0.f), p_on = top_p < 1.f;
    const u64 least = least_weight(min_p);
    const int k = wanted(top_k, vocab);
    const int bits = __clz(vocab) - 1;                     // (as many units of 2^-bits as tokens fit 31 bits)
    // a token's weight into the count of its bin, as find_about reads it: the part of e^(-place / 64) behind the bin's own, e^-in with in < 1/64, by three terms
    const float unit = (float)(1 << bits);
    auto add_about = [&](float at) __attribute__((always_inline)) {
        const float in = __builtin_amdgcn_fractf(at);
        atomicAdd(&s.count[(int)at], (int)fmaf(in, fmaf(in, unit * (0.5f / 4096.f), unit * (-1.f / 64.f)), unit));
    };
    // With top_p alone, or as many wanted as a sort holds, a row that has to be read again is looked through for its largest and for where the cut lies at once: the bins
    // then begin 8 temperatures above the largest of its first logits.  (512 rows of 128000, top_p 0.9: 213 us with a pass for each, 186 so; other steps since: 156.)
    bool anchored = false;
    float anchor = 0.f;
    // With few wanted, or min_p alone, what the first logits rule out is ruled out by all: the others, as far as they find room, are listed while the largest is looked for.
    // (512 rows of 128000, top-k 50 85 us with a reading for each, min-p 88.)
    bool listed = false;
    float m = -INFINITY;
    int lowest = 0;
    if (FOUND) {
        const u64 best = row_best(found_in, r, lane);      // (the same in every wave)
        if (best) m = logit_of(best), lowest = index_of(best);
    } else if (HELD) {
        for (int i0 = 0; i0 < padded; i0 += 16 * NT) {
            float4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = i0 + (k * NT + tid) * 4;
                if (i < padded) v[k] = from_memory(i);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = i0 + (k * NT + tid) * 4;
                if (i >= padded) continue;
                *(float4*)(held + i) = v[k];
                m = fmaxf(m, fmaxf(fmaxf(v[k].x, v[k].y), fmaxf(v[k].z, v[k].w)));
            }
        }
    } else if (!greedy && (k ? k <= NT - NT / 8 : p_on || min_p > 0.f)) {
        float first = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = (j * NT + tid) * 4;
            if (i + 4 <= vocab) {
                const float4 v = from_memory(i);
                first = fmaxf(first, fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)));
            }
        }
        const float own_first = first;
        first = wave_max(first);
        if (lane == 0) s.wave_sum[wave] = __float_as_uint(first);
        if (tid == 0) s.n_list = 0;
        for (int i = tid; i < SAMPLE_BINS; i += NT) s.count[i] = 0;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) first = fmaxf(first, __uint_as_float((unsigned)s.wave_sum[w]));
        anchor = 0.5f * first + 4.f * temperature;        // (half of it)
        anchored = fabsf(anchor) < 0x1p126f;              // (nor does a difference from it overflow)
        const SampleRow from(0.f, temperature);
        float end = 0.f;
        if (anchored && (k ? k <= NT / 4 : !p_on)) {
            anchored = false;
            anchor = 0.5f * first;
            if (k) {                                       // the k-th of the threads' own largest is no larger than the k-th of all
                const float b = from.place_below(anchor, own_first);
                if (b < (float)SAMPLE_BINS) atomicAdd(&s.count[(int)b], 1);
                __syncthreads();
                find_bin<NT, false>(s, true, (u64)k, 0, 0);
                end = (float)(s.found + 1);
            } else {                                       // (with a margin for the roundings)
                end = 64.f * 1.0001f * reach_of_least(least) + 1.f;
            }
            // (not where so many threads' tokens pass that all will not find room: 104 us instead of 111 with min_p 1e-3)
            const int pass = __syncthreads_count(from.place_below(anchor, own_first) < end);
            listed = pass > 0 && (long)pass * vocab <= (long)LIST * 16 * NT;
        }
        if (listed) {
            all_of([&](float v, int i) {
                m = fmaxf(m, v);
                if (from.place_below(anchor, v) < end) {
                    const int at = atomicAdd(&s.n_list, 1);
                    if (at < LIST) s.list[at] = composite(v, i);
                }
            });
        } else if (anchored) {
            all_of([&](float v, int) {
                m = fmaxf(m, v);
                const float at = from.place_below(anchor, v);
                if (!(at < (float)SAMPLE_BINS)) return;
                if (k) atomicAdd(&s.count[(int)fmaxf(at, 0.f)], 1);
                else add_about(fmaxf(at, 0.f));
            });
        } else {
            all_of([&](float v, int) { m = fmaxf(m, v); });
        }
        __syncthreads();
    } else if (greedy) {
        all_of([&](float v, int i) { if (v > m) m = v, lowest = i; });
    } else {
        all_of([&](float v, int) { m = fmaxf(m, v); });
    }
    const float own_top = m;
    m = wave_max(m);
    if (lane == 0) s.wave_sum[wave] = __float_as_uint(m);
    if (tid == 0) s.lowest = 0;
    if (tid == 0 && !listed) s.n_list = 0;
    for (int i = tid; i < SAMPLE_BINS; i += NT) {
        s.sum[i] = 0;
        if (!anchored) s.count[i] = 0;
    }
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, __uint_as_float((unsigned)s.wave_sum[w]));
    if (top == -INFINITY) {
        if (tid == 0) out(-1, 0, 0.f);
        return;
    }
    if (greedy) {                                          // the lowest index of the largest
        if (HELD && !FOUND) all_of([&](float v, int i) { if (v == top) atomicMax(&s.lowest, composite(0.f, i)); });
        else if (own_top == top) atomicMax(&s.lowest, composite(0.f, lowest));
        __syncthreads();
        if (tid == 0) out(index_of(s.lowest), 1, 1.f);
        return;
    }
    infinite = top == INFINITY;
    if (infinite) {
        top = 0.f;
        if (HELD) {
            for (int i = tid; i < padded; i += NT) held[i] = held[i] == INFINITY ? 0.f : -INFINITY;
            __syncthreads();
        }
    }
    const SampleRow row(top, temperature);
    auto weight = [&](float v) __attribute__((always_inline)) -> u64 { return row.weight(v); };
    auto place = [&](float v) -> float { return row.place(v); };
    auto limit_of = [&](u64 sum) -> u64 { return top_p > 0.f ? (u64)ceil((double)top_p * (double)sum) : 1ull; };
    auto place_in = [&](u64 all) -> u64 {
        const u64 t = (u64)floor((double)fminf(fmaxf(u, 0.f), 1.f) * (double)all);
        return t < all ? t : all - 1;
    };
    // the list, one token a thread, holds all that can be kept: sorted, cut, sorted by index and drawn from
    auto draw_listed = [&](int n, bool by_count, u64 total) __attribute__((always_inline)) -> bool {
        u64 e = tid < n ? s.list[tid] : 0;
        __syncthreads();
        e = block_sort(s, e, n);
        u64 w = tid < n && !(by_count && tid >= k) ? weight(logit_of(e)) : 0, all;
        const u64 before = block_scan(s, w, &all) - w;
        if (by_count) total = all;
        else if (all < limit_of(total)) return false;        // (uniform) the cut lies behind what is listed
        const bool keep = w >= least && (!p_on || tid == 0 || before < limit_of(total));
        const int kept = __syncthreads_count(keep);
        u64 o = keep ? ~((u64)index_of(e) << 41 | w) : 0;    // (weights have 41 bits, indices 22)
        o = block_sort(s, o, by_count ? min(n, k) : n);
        w = o ? ~o & ((1ull << 41) - 1) : 0;
        const u64 upto = block_scan(s, w, &all), t = place_in(all);
        if (upto - w <= t && t < upto) out((int)(~o >> 41), kept, (float)((double)w / (double)all));
        return true;
    };
    if (listed) {
        int n = s.n_list;
        if (!infinite && n > NT && n <= LIST) {            // by the row's own largest now
            u64 e[LIST / NT];
            float end = SAMPLE_REACH;
#pragma unroll
            for (int j = 0; j < LIST / NT; ++j) {
                e[j] = j * NT + tid < n ? s.list[j * NT + tid] : 0;
                const float b = place(logit_of(e[j]));
                if (k && e[j] && b < SAMPLE_REACH) atomicAdd(&s.count[(int)b], 1);
            }
            __syncthreads();
            if (tid == 0) s.n_list = 0;
            if (k) {
                find_bin<NT, false>(s, true, (u64)k, 0, 0);
                if (s.found >= 0) end = (float)(s.found + 1);
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < LIST / NT; ++j)
                if (e[j] && (k ? place(logit_of(e[j])) < end : weight(logit_of(e[j])) >= least)) {
                    const int at = atomicAdd(&s.n_list, 1);
                    if (at < NT) s.list[at] = e[j];
                }
            __syncthreads();
            n = s.n_list;
        }
        if (!infinite && n <= NT) {
            draw_listed(n, k > 0, 0);
            return;
        }
        __syncthreads();
        if (tid == 0) s.n_list = 0;
        for (int i = tid; i < SAMPLE_BINS; i += NT) s.count[i] = 0;
        __syncthreads();
    }
    u64 cut = 0;                                           // kept: composites from here on
    // What is kept of each chunk of the row, to s.sum; a wave's share is n_chunks of them, so that a thread has few tokens to go through where the place is.
    // Returns how many tokens this thread saw that are.
    constexpr int UNIT = HELD ? 256 : FOUND ? SAMPLE_CHUNK : 1024, CHUNKS = HELD ? 1 : SAMPLE_BINS / NW;
    const int per_wave = (vocab + NW - 1) / NW, chunk = ((per_wave + CHUNKS - 1) / CHUNKS + UNIT - 1) / UNIT * UNIT, n_chunks = (per_wave + chunk - 1) / chunk;
    auto sum_chunks = [&](auto&& kept_of) __attribute__((always_inline)) -> int {
        const int mine = wave * n_chunks * chunk;
        int n = 0;
        __syncthreads();
        for (int j = 0; j < n_chunks; ++j) {
            u64 sum = 0;
            each(std::integral_constant<int, 64>{}, mine + j * chunk, min(mine + (j + 1) * chunk, padded), lane, [&](float v, int i) {
                const u64 w = kept_of(v, i);
                sum += w;
                n += w != 0;
            });
            sum = wave_scan(sum);
            if (lane == 63) s.sum[wave * n_chunks + j] = sum;
        }
        __syncthreads();
        return n;
    };
    bool summed = false;
    int n_kept = 0;
    if (k || p_on) {
        auto clear = [&]() __attribute__((always_inline)) {
            __syncthreads();
            for (int i = tid; i < SAMPLE_BINS; i += NT) s.sum[i] = 0, s.count[i] = 0;
            __syncthreads();
        };
        auto weigh_bins = [&](bool count) __attribute__((always_inline)) {
            all_of([&](float v, int i) {
                const float b = place(v);
                if (!(b < SAMPLE_REACH) || (cut && composite(v, i) < cut)) return;
                if (count) atomicAdd(&s.count[(int)b], 1);
                atomicAdd(&s.sum[(int)b], weight(v));
            });
            __syncthreads();
        };
        // tokens of the bins up to b, listed as far as there is room
        auto list_upto = [&](int b) __attribute__((always_inline)) {
            const float end = (float)(b + 1);
            all_of([&](float v, int i) {
                if (place(v) < end) {
                    const int at = atomicAdd(&s.n_list, 1);
                    if (at < LIST) s.list[at] = composite(v, i);
                }
            });
            __syncthreads();
        };
        // the last composite of the list, one token a thread, that is kept with `before` tokens and before_sum before it; what weighs up to it
        auto cut_list = [&](int n, int before, u64 before_sum, bool count_mode, u64 limit, u64* sum_upto) __attribute__((always_inline)) -> u64 {
            u64 e = tid < n ? s.list[tid] : 0, all;
            __syncthreads();
            e = block_sort(s, e, n);
            const u64 w = tid < n ? weight(logit_of(e)) : 0, upto = block_scan(s, w, &all) + before_sum;
            const bool keep = tid < n && (count_mode ? (u64)(before + tid) < limit : tid == 0 || upto - w < limit);
            s.list[tid] = e;
            const int kept = __syncthreads_count(keep);
            if (tid == kept - 1) s.lowest = e, s.found_sum = upto;
            __syncthreads();
            *sum_upto = s.found_sum;
            return s.lowest;
        };
        // f(composite) of the tokens of bin b that are not cut off already
        auto of_bin = [&](float b, auto&& f) __attribute__((always_inline)) {
            all_of([&](float v, int i) {
                const float at = place(v);
                if (at >= b && at < b + 1.f && (!cut || composite(v, i) >= cut)) f(composite(v, i));
            });
        };
        // the same for n tokens of bin b, from the list where they fit it: digit by digit of the composite.  The bins are used for it.
        auto cut_digits = [&](float b, int n, int before, u64 before_sum, bool count_mode, u64 limit, u64* sum_upto) __attribute__((always_inline)) -> u64 {
            auto members = [&](auto&& f) __attribute__((always_inline)) {
                if (n <= LIST) {
                    for (int i = tid; i < n; i += NT) f(s.list[i]);
                } else {
                    of_bin(b, f);
                }
                __syncthreads();
            };
            if (tid == 0) s.lowest = ~0ull;
            u64 prefix = 0;
            int shift = 54;
            for (int d = 0; d < 5; ++d) {
                const int bits = d == 2 ? 10 : 11, above = shift;
                shift -= bits;
                clear();
                members([&](u64 e) {
                    if (d > 0 && e >> above != prefix >> above) return;
                    const int bin = (SAMPLE_BINS - 1) - (int)(e >> shift & ((1 << bits) - 1));
                    atomicAdd(&s.count[bin], 1);
                    atomicAdd(&s.sum[bin], weight(logit_of(e)));
                });
                find_bin<NT, true>(s, count_mode, limit, before, before_sum);
                prefix |= (u64)(SAMPLE_BINS - 1 - s.found) << shift;
                before = s.found_before, before_sum = s.found_before_sum;
                *sum_upto = before_sum + s.found_sum;
                if (s.found_count == 1 || (count_mode && (u64)(before + s.found_count) == limit)) break;       // all of the bin
            }
            members([&](u64 e) { if (e >> shift == prefix >> shift) atomicMin(&s.lowest, e); });       // (tokens of other bins may lie above the prefix)
            return s.lowest;
        };
        if (FOUND) {
            for (int i = tid; i < SAMPLE_BINS; i += NT) s.sum[i] = found_in.sum[r * SAMPLE_BINS + i], s.count[i] = found_in.count[r * (SAMPLE_BINS + 1) + i];
            __syncthreads();
        }
        u64 total = 0;
        bool by_count = k > 0;
        // The top_k-th largest of the threads' own largest is no larger than the top_k-th of all: with few wanted, what lies from its bin on is listed without
        // counting all tokens, and most often fits the list.
        if (!FOUND && by_count && k <= NT / 4) {
            const float b = place(infinite ? (own_top == INFINITY ? 0.f : -INFINITY) : own_top);
            if (b < SAMPLE_REACH) atomicAdd(&s.count[(int)b], 1);
            __syncthreads();
            find_bin<NT, false>(s, true, (u64)k, 0, 0);
            const int found = s.found;
            if (found >= 0) {
                list_upto(found);
                const int n = s.n_list;
                if (n <= NT) {
                    draw_listed(n, true, 0);
                    return;
                }
            }
            clear();
            if (tid == 0) s.n_list = 0;
        }
        if (by_count && anchored) {                        // as many as are wanted, and few more, where the bins from the anchor on say
            const bool told = !infinite;
            if (told) find_bin<NT, false>(s, true, (u64)k, 0, 0);
            const int few = s.found_before + s.found_count;
            if (told && s.found >= 0 && few <= NT) {
                const float end = (float)(s.found + 1);
                all_of([&](float v, int i) {
                    if (row.place_below(anchor, v) < end) s.list[atomicAdd(&s.n_list, 1)] = composite(v, i);
                });
                __syncthreads();
                draw_listed(few, true, 0);
                return;
            }
            anchored = false;
            clear();
        }
        if (by_count) {
            if (!FOUND) {
                all_of([&](float v, int) {
                    const float b = place(v);
                    if (b < SAMPLE_REACH) atomicAdd(&s.count[(int)b], 1);
                });
                __syncthreads();
            }
            find_bin<NT, false>(s, true, (u64)k, 0, 0);
            by_count = s.found >= 0;
            if (!by_count && p_on) clear();
        }
        if (!by_count && p_on) {
            // Where the cut lies, by masses to a few parts in 2^bits (or, from the row's pieces, by weights): then one pass weighs all tokens, and each exactly once; it finds
            // out whether that was right.
            const bool known = FOUND && !k;
            float upto;
            int last;
            if (known) {
                u64 mine = 0;
                for (int i = tid; i < SAMPLE_BINS; i += NT) mine += s.sum[i];
                block_scan(s, mine, &total);
                find_bin<NT, true>(s, false, limit_of(total), 0, 0);
                upto = (float)((double)(s.found_before_sum + s.found_sum) / (double)SAMPLE_ONE);
                last = s.found;
            } else {
                if (!anchored || infinite) {
                    if (anchored) clear();
                    all_of([&](float v, int) {
                        const float b = place(v);
                        if (b < SAMPLE_REACH) add_about(b);
                    });
                    __syncthreads();
                }
                upto = find_about<NT>(s, top_p, bits, &last);
            }
            const int found = s.found;
            const bool by_anchor = anchored && !infinite;
            // (what lies as far below the largest weighs nothing from the anchor on either)
            const float half = by_anchor ? anchor : row.half, reach = by_anchor ? fmaxf(row.place_below(anchor, top), 0.f) + SAMPLE_REACH : SAMPLE_REACH;
            auto spot = [&](float v) __attribute__((always_inline)) -> float { return row.place_below(half, v); };
            u64 before_sum = known ? s.found_before_sum : 0, weighed = 0;
            // each token of the bins up to this one weighs about e^-((found + 1) / 64) at least, which says that few can be kept; else what lies before the bin
            // is summed up and its own tokens are listed
            if (upto * __expf((float)(last + 1) * (1.f / 64.f)) < 0.9f * NT) {
                if (known) list_upto(found);
                else {
                    const float end = (float)(last + 1);
                    all_of([&](float v, int i) {
                        const float at = spot(v);
                        if (!(at < reach)) return;
                        weighed += weight(v);
                        if (at < end) {
                            const int to = atomicAdd(&s.n_list, 1);
                            if (to < LIST) s.list[to] = composite(v, i);
                        }
                    });
                    block_scan(s, weighed, &total);
                    __syncthreads();
                }
                const int n = s.n_list;
                if (n <= NT && draw_listed(n, false, total)) return;
            } else {
                const float b = found ? (float)found : -INFINITY;        // (the first bin: from anywhere on; its end is 1)
                const float b_end = (float)(last + 1);
                u64 ahead = 0;
                n_kept = sum_chunks([&](float v, int i) __attribute__((always_inline)) -> u64 {
                    const float at = spot(v);
                    if (!(at < (known ? b_end : reach))) return 0;
                    const bool before = at < b;
                    if (!before && at < b_end) {
                        const int to = atomicAdd(&s.n_list, 1);
                        if (to < LIST) s.list[to] = composite(v, i);
                    }
                    if (known && !before) return 0;
                    const u64 w = weight(v);
                    weighed += w;
                    if (!before) return 0;
                    if (least == 1) return w;
                    ahead += w;
                    return w >= least ? w : 0;
                });
                const int n = s.n_list;
                if (!known) {
                    if (least == 1)
                        for (int i = tid; i < NW * n_chunks; i += NT) ahead += s.sum[i];
                    block_scan(s, weighed, &total);
                    block_scan(s, ahead, &before_sum);
                }
                const u64 limit = limit_of(total);
                if (n <= LIST) {
                    u64 of_bin_sum = 0, mine = 0, unused;
                    for (int i = tid; i < n; i += NT) mine += weight(logit_of(s.list[i]));
                    block_scan(s, mine, &of_bin_sum);
                    if (before_sum < limit && limit <= before_sum + of_bin_sum) {
                        if (n <= NT) cut = cut_list(n, 0, before_sum, false, limit, &unused);
                        else {                             // (the chunks' sums lie where the digits are counted)
                            u64 sums[SAMPLE_BINS / NT];
#pragma unroll
                            for (int j = 0; j < SAMPLE_BINS / NT; ++j) sums[j] = s.sum[j * NT + tid];
                            cut = cut_digits((float)found, n, 0, before_sum, false, limit, &unused);
#pragma unroll
                            for (int j = 0; j < SAMPLE_BINS / NT; ++j) s.sum[j * NT + tid] = sums[j];
                            __syncthreads();
                        }
                        for (int i = tid; i < n; i += NT) {
                            const u64 e = s.list[i], w = e >= cut ? weight(logit_of(e)) : 0;
                            if (w >= least) {
                                ++n_kept;
                                atomicAdd(&s.sum[index_of(e) / chunk], w);
                            }
                        }
                        __syncthreads();
                        summed = true;
                    }
                }
            }
            if (!summed) {                                 // by weights and with counts, the list empty
                __syncthreads();
                if (tid == 0) s.n_list = 0;
                clear();
                weigh_bins(true);
                u64 mine = 0;
                for (int i = tid; i < SAMPLE_BINS; i += NT) mine += s.sum[i];
                block_scan(s, mine, &total);
                find_bin<NT, true>(s, false, limit_of(total), 0, 0);
            }
        } else if (by_count) {
            const int few = s.found_before + s.found_count;
            if (few <= NT) {
                list_upto(s.found);
                draw_listed(few, true, total);
                return;
            }
        }
        if (!summed && (by_count || p_on)) {
            // the last composite that is kept, the cut lying in the bin that was found
            auto find_cut = [&](bool count_mode, u64 limit, u64* sum_upto) __attribute__((always_inline)) -> u64 {
                const float b = (float)s.found;
                const int n = s.found_count, before = s.found_before;
                const u64 before_sum = s.found_before_sum;
                __syncthreads();
                if (tid == 0) s.n_list = 0;
                __syncthreads();
                if (n <= LIST) of_bin(b, [&](u64 e) { s.list[atomicAdd(&s.n_list, 1)] = e; });
                __syncthreads();
                if (n <= NT) return cut_list(n, before, before_sum, count_mode, limit, sum_upto);
                return cut_digits(b, n, before, before_sum, count_mode, limit, sum_upto);
            };
            if (by_count) {
                clear();
                weigh_bins(true);
                find_bin<NT, true>(s, true, (u64)k, 0, 0);
                cut = find_cut(true, (u64)k, &total);
                if (p_on) {                                // the cut by weight lies before the one by count
                    clear();
                    weigh_bins(true);
                    find_bin<NT, true>(s, false, limit_of(total), 0, 0);
                }
            }
            if (p_on) {
                u64 unused;
                const u64 other = find_cut(false, limit_of(total), &unused);
                cut = cut > other ? cut : other;
            }
        }
    }
    // what is kept, a share of the row a wave; then the share that holds the place, a stretch of it a thread.  `bar`: nothing below it is kept (for min_p with a
    // margin for the roundings of its own; the weight decides).
    const float cut_at = cut ? logit_of(cut) : -INFINITY;
    const int cut_index = cut ? index_of(cut) : 0;
    float bar = cut_at;
    if (least > 1) {
        const float low = top - 1.0001f * temperature * reach_of_least(least) - 1e-6f * fabsf(top);
        if (low <= top) bar = fmaxf(bar, low);
    }
    auto kept_weight = [&](float v, int i) __attribute__((always_inline)) -> u64 {
        if (!(v >= bar) || (cut && v == cut_at && i > cut_index)) return 0;
        const u64 w = weight(v);
        return w >= least ? w : 0;
    };
    if (FOUND && !k && !p_on) {
        for (int i = tid; i < SAMPLE_BINS; i += NT) s.sum[i] = found_in.sum[r * SAMPLE_BINS + i];
        if (tid == 0) n_kept = found_in.count[r * (SAMPLE_BINS + 1) + SAMPLE_BINS];
        __syncthreads();
    } else if (!summed) {
        if (!cut && least == 1) n_kept = sum_chunks([&](float v, int) __attribute__((always_inline)) -> u64 { return weight(v); });      // (19 of 133 us for 512 rows of 128000)
        else n_kept = sum_chunks(kept_weight);
    }
    int kept;
    u64 all;
    block_scan(s, n_kept, &kept);
    __syncthreads();
    // the chunk that holds the place
    constexpr int PER = SAMPLE_BINS / NT;
    u64 own_sum[PER], mass = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) mass += own_sum[j] = tid * PER + j < NW * n_chunks ? s.sum[tid * PER + j] : 0;
    u64 before = block_scan(s, mass, &all) - mass;
    const u64 t = place_in(all);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        if (before <= t && t < before + own_sum[j]) s.found = tid * PER + j, s.found_before_sum = before;
        before += own_sum[j];
    }
    __syncthreads();
    before = s.found_before_sum;
    const int first = s.found * chunk, end = min(first + chunk, vocab), own = (chunk + NT - 1) / NT;
    const int a = min(first + tid * own, end), b = min(a + own, end);
    auto at = [&](int i) -> float {
        const float v = HELD ? held[i] : x[i];
        return HELD || !infinite ? v : v == INFINITY ? 0.f : -INFINITY;
    };
    u64 here = 0;
    for (int i = a; i < b; ++i) here += kept_weight(at(i), i);
    u64 unused;
    u64 upto = block_scan(s, here, &unused) + before;
    if (upto - here <= t && t < upto) {
        upto -= here;
        for (int i = a; i < b; ++i) {
            const u64 w = kept_weight(at(i), i);
            upto += w;
            if (t < upto) {
                out(i, kept, (float)((double)w / (double)all));
                break;
            }
        }
    }
}
constexpr int SAMPLE_HELD = 32512;         // logits that fit LDS beside the bins
hipError_t launch_sample(const Sample& c, int rows, int vocab, float* ws, size_t ws_elems, hipStream_t s) {
    if (rows <= 0) return hipSuccess;
    SampleFound w{};
    // A row held in LDS, one workgroup to a CU, as long as there are no more rows than CUs; beyond, rows read again by workgroups of 512 threads, two or more to a CU.  us held /
    // read again by 1024 threads / by 512: 256 rows of 32000, top-k 50 16 / 19 / 19, min-p 15 / 19 / 19, top-p 0.9 32 / 34 / 33, top-k 1000 29 / 31 / 46; 257 rows 28 / 31 / 20, 24 / 28 / 18,
    // 59 / 62 / 43, 56 / 58 / 58; 1024 rows 65 / 72 / 45, 58 / 67 / 43, 126 / 132 / 89, 114 / 119 / 127; 256 rows of 128000 - / 38 / 44, - / 39 / 41, - / 85 / 98, - / 115 / 140; 512 rows - / 73 / 58,
    // - / 72 / 58, - / 167 / 148, - / 186 / 217 (more wanted than 512 threads sort: the one side on which 1024 win; the settings are not known here).
    if (vocab <= SAMPLE_HELD && rows <= 256) {
        const int lds = ((vocab + 3) & ~3) * 4;
        const hipError_t e = hipFuncSetAttribute((const void*)sample_kernel<1024, 1024, true, false>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 SAMPLE_HELD * 4);        // (the same from every thread of the host)
        if (e != hipSuccess) return e;
        sample_kernel<1024, 1024, true, false><<<rows, 1024, lds, s>>>(c, vocab, w);
        return hipGetLastError();
    }
    // Few rows of many tokens: pieces of a row on CUs of their own, then a workgroup a row.  us in pieces and in one workgroup, one row of 66000 / 128000 / 262144 / 1000000, 16 of
    // 66000 / 128000 / 262144: no limit 17 and 26 / 18 and 40 / 21 and 73 / 37 and 283, 18 and 26 / 19 and 41 / 27 and 81; min-p 17 and 15 / 17 and 18 / 17 and 26 / 18 and 91, 18 and 16 / 18
    // and 22 / 23 and 36; top-p 0.9 36 and 40 / 46 and 62 / 68 and 111 / 193 and 396, 58 and 53 / 83 and 79 / 139 and 144; top-k 50 24 and 18 / 27 and 24 / 34 and 35 / 100 and 167, 24
    // and 19 / 31 and 25 / 45 and 43 (two launches more are 6 us of it; the settings are not known here).
    const size_t at = (uintptr_t)ws & 7 ? 1 : 0;           // (64-bit places in scratch that begins at any multiple of 4)
    w.pieces = cdiv(vocab, SAMPLE_PIECE);
    const size_t need = at + (size_t)rows * (2 * w.pieces + 3 * SAMPLE_BINS + 1);
    if (ws && vocab > 65536 && rows <= 16 && vocab <= SAMPLE_BINS * SAMPLE_CHUNK && need <= ws_elems) {
        w.best = (u64*)(ws + at);
        w.sum = w.best + (size_t)rows * w.pieces;
        w.count = (int*)(w.sum + (size_t)rows * SAMPLE_BINS);
        const dim3 grid(w.pieces, rows);
        sample_best_kernel<<<grid, 1024, 0, s>>>(c, vocab, w);
        sample_weigh_kernel<<<grid, 1024, 0, s>>>(c, vocab, w);
        sample_kernel<1024, 2048, false, true><<<rows, 1024, 0, s>>>(c, vocab, w);
        return hipGetLastError();
    }
    if (rows <= 256) sample_kernel<1024, 2048, false, false><<<rows, 1024, 0, s>>>(c, vocab, w);
    else sample_kernel<512, 2048, false, false><<<rows, 512, 0, s>>>(c, vocab, w);
    return hipGetLastError();
}
