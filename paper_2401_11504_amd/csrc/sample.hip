// A token drawn from each row of logits: temperature, top-k, top-p, min-p, and a given number.
//   w_i = round(2^40 exp((x_i - largest) / temperature))      whole numbers, so that sums of them are exact in any order
// The order is that of the logits, the lowest index first among equals.  Kept are the first top_k of it, of these the ones that less than top_p of
// their weight lies before, of these the ones with at least min_p of the largest weight.  With S the kept weight, the token is the first in the order
// of the indices up to which more than floor(u S) is kept.
#include "kernels.h"

typedef unsigned long long u64;
constexpr u64 SAMPLE_ONE = 1ull << 40;
constexpr int SAMPLE_NT = 1024, SAMPLE_NW = SAMPLE_NT / 64, SAMPLE_BINS = 2048, SAMPLE_LIST = 4096;

// 2^y in units of 2^-40, y <= 0, rounded to the nearest: 2^n e^(f ln 2) with y = n + f, |f| <= 1/2, the exponential by its series up to the 13th power
// (the first term left out is below 2^-57).  Adding 2^52 rounds to a whole number and leaves it in the mantissa's low bits.
__device__ __forceinline__ u64 weight_of(double y) {
    if (!(y > -41.5)) return 0;
    const double n = rint(y), t = (y - n) * 0.693147180559945309417;
    double p = 1.0 / 6227020800.0;
    p = fma(p, t, 1.0 / 479001600.0);
    p = fma(p, t, 1.0 / 39916800.0);
    p = fma(p, t, 1.0 / 3628800.0);
    p = fma(p, t, 1.0 / 362880.0);
    p = fma(p, t, 1.0 / 40320.0);
    p = fma(p, t, 1.0 / 5040.0);
    p = fma(p, t, 1.0 / 720.0);
    p = fma(p, t, 1.0 / 120.0);
    p = fma(p, t, 1.0 / 24.0);
    p = fma(p, t, 1.0 / 6.0);
    p = fma(p, t, 0.5);
    p = fma(p, t, 1.0);
    p = fma(p, t, 1.0);
    const double scale = __longlong_as_double((long long)((int)n + 40 + 1023) << 52);
    return (u64)__double_as_longlong(fma(p, scale, 4503599627370496.0)) & 0xfffffffffffffull;
}
// larger for larger x, the same for 0 and -0
__device__ __forceinline__ unsigned key_of_logit(float x) {
    const unsigned u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of_key(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

struct SampleRow {
    float top, bins;                      // the largest logit; bins of a unit of x
    double per;                           // log2(e) / temperature
    __device__ __forceinline__ u64 weight(float x) const { return x == top ? SAMPLE_ONE : weight_of(((double)x - (double)top) * per); }
    // a coarse place in the order, 0 for the largest: monotone, as every step of it is
    __device__ __forceinline__ int bin(float x) const { return x == top ? 0 : (int)fminf((top - x) * bins, (float)(SAMPLE_BINS - 1)); }
    __device__ __forceinline__ bool counts(float x) const { return x == top || ((double)x - (double)top) * per > -41.5; }       // may weigh something (NaN: no)
};

// f(x[i], i) for first <= i < end, the workgroup's (or a wave's) lanes side by side
template <int LANES, int U, class F>
__device__ __forceinline__ void each_logit(const float* x, int first, int end, int lane, F&& f) {
    for (int i0 = first; i0 < end; i0 += 4 * LANES * U) {
        float4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + (u * LANES + lane) * 4;
            if (i + 4 <= end) v[u] = *(const float4*)(x + i);
            else {
#pragma unroll
                for (int e = 0; e < 4; ++e) (&v[u].x)[e] = i + e < end ? x[i + e] : -INFINITY;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + (u * LANES + lane) * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < end) f((&v[u].x)[e], i + e);
        }
    }
}

struct SampleLds {
    u64 sum[SAMPLE_BINS];
    int count[SAMPLE_BINS];
    u64 list[SAMPLE_LIST];
    u64 wave_sum[SAMPLE_NW];
    int wave_count[SAMPLE_NW];
    u64 found_sum, found_before_sum, lowest;
    int found, found_count, found_before, n_list;
};
// inclusive sums over the threads of the workgroup; the total to *all
__device__ __forceinline__ u64 block_scan(SampleLds& s, u64 v, u64* all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const u64 o = __shfl_up(v, off, 64);
        if (lane >= off) v += o;
    }
    __syncthreads();
    if (lane == 63) s.wave_sum[wave] = v;
    __syncthreads();
    u64 total = 0;
#pragma unroll
    for (int w = 0; w < SAMPLE_NW; ++w) {
        if (w < wave) v += s.wave_sum[w];
        total += s.wave_sum[w];
    }
    *all = total;
    return v;
}
__device__ __forceinline__ int block_count(SampleLds& s, int v) {
    u64 all;
    block_scan(s, (u64)v, &all);
    return (int)all;
}
__device__ __forceinline__ void clear_bins(SampleLds& s) {
    for (int i = threadIdx.x; i < SAMPLE_BINS; i += SAMPLE_NT) s.sum[i] = 0, s.count[i] = 0;
    __syncthreads();
}
// the bin in which the count (by_count) or the weight, summed up from bin 0 and on top of before_*, first reaches `limit`: s.found (-1: none does), its own
// count and sum, and those before it
__device__ __forceinline__ void find_bin(SampleLds& s, bool by_count, u64 limit, int before_count, u64 before_sum) {
    const int b = 2 * threadIdx.x;
    u64 all;
    __syncthreads();
    if (threadIdx.x == 0) s.found = -1;
    const int c0 = s.count[b], c1 = s.count[b + 1];
    const u64 w0 = s.sum[b], w1 = s.sum[b + 1];
    const int c = (int)block_scan(s, (u64)(c0 + c1), &all) + before_count;
    const u64 w = block_scan(s, w0 + w1, &all) + before_sum;
    auto take = [&](int at, int n, u64 x, int nb, u64 xb) { s.found = at, s.found_count = n, s.found_sum = x, s.found_before = nb, s.found_before_sum = xb; };
    const u64 end = by_count ? (u64)c : w, mid = by_count ? (u64)(c - c1) : w - w1, start = by_count ? (u64)(c - c0 - c1) : w - w0 - w1;
    if (start < limit && limit <= mid) take(b, c0, w0, c - c0 - c1, w - w0 - w1);
    if (mid < limit && limit <= end) take(b + 1, c1, w1, c - c1, w - w1);
    __syncthreads();
}
// one value a thread, the largest in thread 0
__device__ __forceinline__ u64 block_sort(SampleLds& s, u64 v, int n) {
    int size = 64;
    while (size < n) size <<= 1;
    const int t = threadIdx.x;
    for (int k = 2; k <= size; k <<= 1) {
        for (int j = k >> 1; j > 0; j >>= 1) {
            u64 o;
            if (j < 64) o = __shfl_xor(v, j, 64);
            else {
                __syncthreads();
                s.list[t] = v;
                __syncthreads();
                o = s.list[t ^ j];
            }
            const bool larger = ((t & k) == 0) == ((t & j) == 0);      // this one keeps the larger
            v = larger ? (v > o ? v : o) : (v < o ? v : o);
        }
    }
    return v;
}

__global__ __launch_bounds__(SAMPLE_NT) void sample_kernel(Sample c, int vocab) {
    __shared__ SampleLds s;
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

    // the largest, and its lowest index for the choice without a temperature
    float m = -INFINITY;
    int at = 0x7fffffff;
    const bool greedy = !(temperature > 0.f);
    if (greedy) each_logit<SAMPLE_NT, 4>(x, 0, vocab, tid, [&](float v, int i) { if (v > m) m = v, at = i; });
    else each_logit<SAMPLE_NT, 4>(x, 0, vocab, tid, [&](float v, int) { m = fmaxf(m, v); });
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const float o = __shfl_xor(m, off, 64);
        const int oi = __shfl_xor(at, off, 64);
        if (o > m || (o == m && oi < at)) m = o, at = oi;
    }
    if (lane == 0) s.wave_sum[wave] = (u64)key_of_logit(m) << 32 | (unsigned)~at;
    __syncthreads();
    u64 best = 0;
#pragma unroll
    for (int w = 0; w < SAMPLE_NW; ++w) best = best > s.wave_sum[w] ? best : s.wave_sum[w];
    __syncthreads();
    SampleRow row;
    row.top = logit_of_key((unsigned)(best >> 32));
    if (row.top == -INFINITY) {
        if (tid == 0) out(-1, 0, 0.f);
        return;
    }
    if (greedy) {
        if (tid == 0) out((int)~(unsigned)best, 1, 1.f);
        return;
    }
    row.per = 1.0 / (double)temperature * 1.44269504088896340736;
    row.bins = 64.f / temperature;

    const int k = top_k >= 1.f && top_k < (float)vocab ? (int)top_k : 0;
    const bool p_on = top_p < 1.f;
    u64 least = 1;
    if (min_p > 0.f) least = min_p >= 1.f ? SAMPLE_ONE : (u64)ceil((double)min_p * (double)SAMPLE_ONE);
    auto limit_of = [&](u64 sum) -> u64 { return top_p > 0.f ? (u64)ceil((double)top_p * (double)sum) : 1ull; };
    auto composite = [&](float v, int i) -> u64 { return (u64)key_of_logit(v) << 22 | (unsigned)(0x3fffff - i); };        // larger: earlier in the order
    u64 threshold = 0;                                     // kept: composites from here on
    if (k || p_on) {
        clear_bins(s);
        each_logit<SAMPLE_NT, 4>(x, 0, vocab, tid, [&](float v, int) {
            if (!row.counts(v)) return;
            const int b = row.bin(v);
            atomicAdd(&s.count[b], 1);
            if (p_on) atomicAdd(&s.sum[b], row.weight(v));
        });
        __syncthreads();
        u64 total = 0;
        bool by_count = k > 0;
        if (by_count) {
            find_bin(s, true, (u64)k, 0, 0);
            by_count = s.found >= 0;
        }
        if (!by_count && p_on) {
            block_scan(s, s.sum[2 * tid] + s.sum[2 * tid + 1], &total);
            find_bin(s, false, limit_of(total), 0, 0);
        }
        if (by_count || p_on) {
            const int few = s.found_before + s.found_count;
            if (few <= SAMPLE_NT) {
                // all that can be kept fits one token a thread
                const int b = s.found;
                if (tid == 0) s.n_list = 0;
                __syncthreads();
                each_logit<SAMPLE_NT, 4>(x, 0, vocab, tid, [&](float v, int i) {
                    if (row.counts(v) && row.bin(v) <= b) s.list[atomicAdd(&s.n_list, 1)] = composite(v, i);
                });
                __syncthreads();
                u64 e = tid < few ? s.list[tid] : 0;
                e = block_sort(s, e, few);
                const int i = 0x3fffff - (int)(e & 0x3fffff);
                u64 w = tid < few ? row.weight(logit_of_key((unsigned)(e >> 22))) : 0, all;
                if (by_count && tid >= k) w = 0;
                const u64 before = block_scan(s, w, &all) - w;
                if (by_count) total = all;
                const bool keep = w >= least && (!p_on || tid == 0 || before < limit_of(total));
                const int kept = block_count(s, keep);
                u64 o = keep ? ~((u64)i << 41 | w) : 0;    // (weights have 41 bits, indices 22)
                o = block_sort(s, o, few);
                w = o ? ~o & ((1ull << 41) - 1) : 0;
                const u64 upto = block_scan(s, w, &all);
                u64 t = (u64)floor((double)fminf(fmaxf(u, 0.f), 1.f) * (double)all);
                t = t < all ? t : all - 1;
                if (upto - w <= t && t < upto) out((int)(~o >> 41), kept, (float)((double)w / (double)all));
                return;
            }
            // the place of a cut inside bin b of the coarse order: digit by digit of the composite; its elements from the list if they fit one
            auto cut = [&](bool count_mode, u64 limit, u64* sum_upto) -> u64 {
                const int b = s.found, n = s.found_count;
                int before = s.found_before;
                u64 before_sum = s.found_before_sum;
                const bool listed = n <= SAMPLE_LIST;
                __syncthreads();
                if (tid == 0) s.n_list = 0;
                __syncthreads();
                if (listed) {
                    each_logit<SAMPLE_NT, 4>(x, 0, vocab, tid, [&](float v, int i) {
                        if (row.counts(v) && row.bin(v) == b && composite(v, i) >= threshold) s.list[atomicAdd(&s.n_list, 1)] = composite(v, i);
                    });
                }
                auto each = [&](auto&& f) {
                    if (listed) {
                        for (int i = tid; i < n; i += SAMPLE_NT) f(s.list[i]);
                    } else {
                        each_logit<SAMPLE_NT, 4>(x, 0, vocab, tid, [&](float v, int i) {
                            if (row.counts(v) && row.bin(v) == b && composite(v, i) >= threshold) f(composite(v, i));
                        });
                    }
                    __syncthreads();
                };
                u64 prefix = 0;
                int shift = 54;
                for (int d = 0; d < 5; ++d) {
                    const int bits = d == 2 ? 10 : 11, above = shift;
                    shift -= bits;
                    clear_bins(s);
                    each([&](u64 e) {
                        if (d > 0 && e >> above != prefix >> above) return;
                        const int bin = (SAMPLE_BINS - 1) - (int)(e >> shift & ((1 << bits) - 1));
                        atomicAdd(&s.count[bin], 1);
                        atomicAdd(&s.sum[bin], row.weight(logit_of_key((unsigned)(e >> 22))));
                    });
                    find_bin(s, count_mode, limit, before, before_sum);
                    prefix |= (u64)(SAMPLE_BINS - 1 - s.found) << shift;
                    before = s.found_before, before_sum = s.found_before_sum;
                    *sum_upto = before_sum + s.found_sum;
                    if (s.found_count == 1 || (count_mode && (u64)(before + s.found_count) == limit)) break;       // all of the bin
                }
                // (other coarse bins may lie above the prefix: the cut is the last composite that is kept)
                if (tid == 0) s.lowest = ~0ull;
                __syncthreads();
                each([&](u64 e) { if (e >> shift == prefix >> shift) atomicMin(&s.lowest, e); });
                return s.lowest;
            };
            if (by_count) {
                threshold = cut(true, (u64)k, &total);
                if (p_on) {
                    // the cut by weight lies before the one by count: its bin is found over the coarse bins again
                    clear_bins(s);
                    each_logit<SAMPLE_NT, 4>(x, 0, vocab, tid, [&](float v, int i) {
                        if (!row.counts(v) || composite(v, i) < threshold) return;
                        const int b = row.bin(v);
                        atomicAdd(&s.count[b], 1);
                        atomicAdd(&s.sum[b], row.weight(v));
                    });
                    __syncthreads();
                    find_bin(s, false, limit_of(total), 0, 0);
                }
            }
            if (p_on) {
                u64 unused;
                const u64 limit = limit_of(total), other = cut(false, limit, &unused);
                threshold = threshold > other ? threshold : other;
            }
        }
    }
    // what is kept, a 16th of the row a wave; then the 16th that holds the place, a stretch of it a thread
    const int stretch = ((vocab + SAMPLE_NW - 1) / SAMPLE_NW + 255) & ~255;
    auto weight = [&](float v, int i) -> u64 {
        if (threshold && composite(v, i) < threshold) return 0;
        const u64 w = row.weight(v);
        return w >= least ? w : 0;
    };
    u64 sum = 0;
    int n = 0;
    const int mine = wave * stretch;
    each_logit<64, 4>(x, mine, min(mine + stretch, vocab), lane, [&](float v, int i) {
        const u64 w = weight(v, i);
        sum += w;
        n += w != 0;
    });
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    const int kept = block_count(s, n);
    __syncthreads();
    if (lane == 0) s.wave_sum[wave] = sum;
    __syncthreads();
    u64 all = 0;
#pragma unroll
    for (int w = 0; w < SAMPLE_NW; ++w) all += s.wave_sum[w];
    u64 t = (u64)floor((double)fminf(fmaxf(u, 0.f), 1.f) * (double)all);
    t = t < all ? t : all - 1;
    int part = 0;
    u64 before = 0;
    for (; part < SAMPLE_NW - 1 && before + s.wave_sum[part] <= t; ++part) before += s.wave_sum[part];
    const int first = part * stretch, end = min(first + stretch, vocab), per = stretch / SAMPLE_NT + (stretch % SAMPLE_NT != 0);
    const int a = min(first + tid * per, end), b = min(a + per, end);
    u64 own = 0;
    for (int i = a; i < b; ++i) own += weight(x[i], i);
    u64 unused;
    u64 upto = block_scan(s, own, &unused) + before;
    if (upto - own <= t && t < upto) {
        upto -= own;
        for (int i = a; i < b; ++i) {
            const u64 w = weight(x[i], i);
            upto += w;
            if (t < upto) {
                out(i, kept, (float)((double)w / (double)all));
                break;
            }
        }
    }
}
hipError_t launch_sample(const Sample& c, int rows, int vocab, float* ws, size_t ws_elems, hipStream_t s) {
    if (rows <= 0) return hipSuccess;
    (void)ws, (void)ws_elems;
    sample_kernel<<<rows, SAMPLE_NT, 0, s>>>(c, vocab);
    return hipGetLastError();
}
