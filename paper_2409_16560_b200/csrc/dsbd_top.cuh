// The K largest logits of a row, in one pass over it.
//
// Each CTA of the row's cluster reads its share once, in batches of a few 16-byte words a thread, and keeps nothing but the words with a token that
// may be among the K largest; the others go into the sum of the rest at once.  May be: at or above a bound, the K-th largest of the maxima of 4
// groups of words a thread that have been seen so far (by bins: every one of those K groups has a token that reaches it).  The bound is made from
// a batch before that is looked at, and again when two or four times as many have been seen: as many tokens as were seen before add about 1.4 K
// words.  Kept words are sorted out later, many at a time and against a better bound: their tokens at or above it go to a list, the others to the rest.
// At the end rank 0 takes the others' lists, and sorts.
// Rows with more equal logits at the cut than the list holds are selected by the bits of their keys in passes of their own.
#pragma once

#include "dsbd_rows.cuh"

namespace dsbd {
namespace rows {

constexpr int kBins = 512;

__device__ __forceinline__ float logit_of(uint64_t entry) { return of_key((uint32_t)(entry >> 32)); }
__device__ __forceinline__ int token_of(uint64_t entry) { return (int)~(uint32_t)entry; }
__device__ __forceinline__ uint64_t entry_of(float z, int token) { return ((uint64_t)key_of(z) << 32) | (uint32_t)~token; }

// Number of the bin of width 1 / scale below the largest; falls nowhere as z grows.
__device__ __forceinline__ int bin_below(float top, float z, float scale) {
    return min(__float2int_rz((top - z) * scale), kBins - 1);
}

// Bins that span `width`; none (everything in one) where the width has no finite inverse.
__device__ __forceinline__ float bins_over(float width) {
    const float scale = (float)(kBins - 1) / width;
    return scale < 1e30f ? scale : 0.f;
}

// NT threads, maxima of G groups of words a thread, lists of LIST entries
// and HOT words kept.
template <int NT, int G, int LIST, int HOT>
struct TopList {
    static constexpr int kWarps_ = NT / 32;
    static constexpr int kEach = LIST / NT;        // entries of a thread
    static constexpr int kTop = NT * G / 2;        // K, at most: half the groups
    static_assert(kBins % NT == 0 && LIST % NT == 0 && LIST >= 2 * kTop && HOT * sizeof(float4) >= LIST * sizeof(uint64_t), "");

    static constexpr int kList = LIST;

    float4 hot[HOT];
    int hot_token[HOT];                            // of the word's first element
    uint64_t list[LIST];
    uint32_t count[kBins], scan[kWarps_];
    float high[kWarps_], low[kWarps_];
    double sums[kWarps_];
    uint32_t listed, hots, last;

    // Largest and smallest of the threads' h and l, to all.
    __device__ __forceinline__ void range(float &h, float &l) {
        h = warp_max(h);
        l = -warp_max(-l);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) { high[threadIdx.x / 32] = h; low[threadIdx.x / 32] = l; }
        __syncthreads();
        h = high[0];
        l = low[0];
#pragma unroll
        for (int w = 1; w < kWarps_; ++w) { h = fmaxf(h, high[w]); l = fminf(l, low[w]); }
    }

    // A number at or below the K-th largest of the threads' values above -inf, and no smaller than it has to be by more than a bin;
    // -inf if there are fewer.  each(f): f(value) for this thread's.
    template <class F>
    __device__ __forceinline__ float bound(uint32_t K, F each) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
        float h = -CUDART_INF_F, l = CUDART_INF_F;
        each([&](float x) { if (x > -CUDART_INF_F) { h = fmaxf(h, x); l = fminf(l, x); } });
        for (int b = threadIdx.x; b < kBins; b += NT) count[b] = 0;
        range(h, l);
        if (threadIdx.x == 0) last = kBins;
        const float scale = bins_over(h - l);
        each([&](float x) { if (x > -CUDART_INF_F) atomicAdd(&count[bin_below(h, x, scale)], 1u); });
        __syncthreads();
        constexpr int kPerThread = kBins / NT;
        uint32_t n[kPerThread], sum = 0;
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) sum += n[i] = count[threadIdx.x * kPerThread + i];
        uint32_t up = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(kFull, up, o);
            if (lane >= o) up += x;
        }
        if (lane == 31) scan[warp] = up;
        __syncthreads();
        uint32_t base = up - sum;
#pragma unroll
        for (int w = 0; w < kWarps_; ++w) base += w < warp ? scan[w] : 0;
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            if (base < K && base + n[i] >= K) last = threadIdx.x * kPerThread + i;
            base += n[i];
        }
        __syncthreads();
        const int bin = (int)last;
        if (bin == kBins) return -CUDART_INF_F;
        float none = -CUDART_INF_F;
        l = CUDART_INF_F;
        each([&](float x) { if (x > -CUDART_INF_F && bin_below(h, x, scale) <= bin) l = fminf(l, x); });
        range(none, l);
        return l;
    }

    // The same of the list's entries.
    __device__ __forceinline__ float entries_bound(uint32_t K) {
        return bound(K, [&](auto f) {
            for (int i = threadIdx.x; i < (int)listed; i += NT) f(logit_of(list[i]));
        });
    }

    // Clears the list of entries below `least`, whose sum goes to `cleared`, the same in all threads.  The list has its tokens in no order,
    // so the terms are made multiples of 2^-40 of the largest: their sum has no roundings that could depend on one.  All threads,
    // behind a barrier.
    template <bool REST>
    __device__ __forceinline__ void clear(float least, float scale, Sum &cleared) {
        const uint32_t n = listed, key = key_of(least);
        static_assert(kEach <= 16 && LIST <= 1 << (53 - 40), "");
        uint64_t e[kEach];
        float h = -CUDART_INF_F, l = 0.f;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            e[i] = threadIdx.x + i * NT < n ? list[threadIdx.x + i * NT] : 0;
            if (e[i] && (uint32_t)(e[i] >> 32) < key) h = fmaxf(h, logit_of(e[i]));
        }
        if (REST) range(h, l);                     // (barriers)
        else __syncthreads();
        if (threadIdx.x == 0) listed = 0;
        __syncthreads();
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (e[i] == 0) continue;
            if ((uint32_t)(e[i] >> 32) >= key) list[next_place(&listed)] = e[i];
            else if (REST) sum += rint((double)exp2_fast((logit_of(e[i]) - h) * scale) * 0x1p40);
        }
        if (!REST) {
            __syncthreads();
            return;
        }
        sum = warp_sum(sum);
        if ((threadIdx.x & 31) == 0) sums[threadIdx.x / 32] = sum;
        __syncthreads();
        if (h == -CUDART_INF_F) return;
        sum = 0.0;
        for (int w = 0; w < kWarps_; ++w) sum += sums[w];
        cleared.add({h, sum * 0x1p-40}, scale);
    }

    // The kept words' tokens at or above `least` to the list, the others' sum to `cleared` (as in clear; of more terms, so in steps of 2^-38).
    template <class T, bool REST>
    __device__ __forceinline__ void flush(float least, float scale, Sum &cleared) {
        constexpr int P = kPer<T>;
        static_assert((uint64_t)HOT * P <= 1ull << (53 - 38), "sums of whole numbers are exact");
        const int n = (int)hots;
        float h = -CUDART_INF_F, l = 0.f;
        for (int i = threadIdx.x; i < n; i += NT) {
            float x[P];
            unpack(hot[i], x);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                if (x[e] >= least) {
                    const uint32_t to = next_place(&listed);
                    if (to < (uint32_t)LIST) list[to] = entry_of(x[e], hot_token[i] + e);
                } else {
                    h = fmaxf(h, x[e]);
                }
            }
        }
        if (!REST) {
            __syncthreads();
            if (threadIdx.x == 0) hots = 0;
            __syncthreads();
            return;
        }
        range(h, l);                               // (barriers)
        const float from = h == -CUDART_INF_F ? 0.f : h;
        double sum = 0.0;
        for (int i = threadIdx.x; i < n; i += NT) {
            float x[P];
            unpack(hot[i], x);
#pragma unroll
            for (int e = 0; e < P; ++e)
                if (x[e] < least) sum += rint((double)exp2_fast((x[e] - from) * scale) * 0x1p38);
        }
        sum = warp_sum(sum);
        if ((threadIdx.x & 31) == 0) sums[threadIdx.x / 32] = sum;
        __syncthreads();
        if (threadIdx.x == 0) hots = 0;
        sum = 0.0;
        for (int w = 0; w < kWarps_; ++w) sum += sums[w];
        cleared.add({h, sum * 0x1p-38}, scale);
        __syncthreads();
    }

    // The list in falling order.
    __device__ __forceinline__ void sort() {
        const int n = (int)listed;
        if (n <= NT && n <= 128) {
            // by rank: how many entries are larger
            const uint64_t e = (int)threadIdx.x < n ? list[threadIdx.x] : 0;
            int rank = 0;
            if ((int)(threadIdx.x & ~31u) < n)
                for (int k = 0; k < n; ++k) rank += list[k] > e;
            __syncthreads();
            if (e) list[rank] = e;
            __syncthreads();
        } else {
            float h = -CUDART_INF_F, l = CUDART_INF_F;
            for (int i = threadIdx.x; i < n; i += NT) {
                const float z = logit_of(list[i]);
                h = fmaxf(h, z);
                l = fminf(l, z);
            }
            range(h, l);
            const float scale = bins_over(h - l);
            order_down<NT, kBins>(list, reinterpret_cast<uint64_t *>(hot), n, count, scan, [&](uint64_t e) { return bin_below(h, logit_of(e), scale); });
        }
    }
};

// Collects the share's tokens at or above the K-th largest logit (and few more, or, of equal ones, many) in the list; REST: the others' sum,
// each thread's in `rest`.  False for a NaN or +inf.  The list may have run over (listed > LIST): then it and the rest are of no use.
template <class T, bool REST, int NT, int G, int LIST, int HOT>
__device__ __forceinline__ bool collect(TopList<NT, G, LIST, HOT> &sh, const T *row, const Share &s, uint32_t K, bool trim, float scale, Rest &rest, Sum &cleared) {
    constexpr int P = kPer<T>, D = kDeep<T>;
    static_assert(D % G == 0, "");
    float group[G], bound = -CUDART_INF_F;
#pragma unroll
    for (int g = 0; g < G; ++g) group[g] = -CUDART_INF_F;
    auto groups = [&](auto f) {
#pragma unroll
        for (int g = 0; g < G; ++g) f(group[g]);
    };
    if (threadIdx.x == 0) sh.listed = sh.hots = 0;
    // behind a barrier: the words kept so far; once they or the list have run over, nothing more
    auto sort_out = [&] {
        const uint32_t hots = sh.hots, listed = sh.listed;
        __syncthreads();
        if (hots > HOT || listed > LIST) {
            if (threadIdx.x == 0) sh.listed = LIST + 1;
            __syncthreads();
        } else {
            if (listed > LIST / 2) sh.template clear<REST>(bound, scale, cleared);
            sh.template flush<T, REST>(bound, scale, cleared);
        }
    };
    int batch = 0, next = 0;
    for (int w0 = 0; w0 < s.words; w0 += D * NT, ++batch) {
        float4 raw[D];
        load_batch<T, NT>(raw, row, s, w0);
        float most[D], top = -CUDART_INF_F;
#pragma unroll
        for (int u = 0; u < D; ++u) {
            float x[P];
            unpack(raw[u], x);
            most[u] = x[0];
#pragma unroll
            for (int e = 1; e < P; ++e) most[u] = max_nan(most[u], x[e]);
            group[u % G] = max_nan(group[u % G], most[u]);
        }
        if (batch == next) {
            bound = fmaxf(sh.bound(K, groups), -FLT_MAX);
            if (batch) sort_out();
            next = max(4 * K <= NT * G ? 4 * next : 2 * next, 1);
        }
#pragma unroll
        for (int u = 0; u < D; ++u) {
            if (most[u] >= bound) {
                const uint32_t to = next_place(&sh.hots);
                if (to < (uint32_t)HOT) {
                    sh.hot[to] = raw[u];
                    sh.hot_token[to] = s.first + batch_word<D>(w0, u) * P - s.mis;
                }
                raw[u] = masked_word<T>();
                most[u] = -CUDART_INF_F;
            }
            top = fmaxf(top, most[u]);
        }
        if (REST) rest.add_words<T>(raw, top, scale);
    }
    // a list that goes to another CTA holds little more than K
    if (batch > 1) bound = fmaxf(sh.bound(K, groups), -FLT_MAX);
    __syncthreads();
    sort_out();
    if (trim && sh.listed <= LIST) sh.template clear<REST>(bound, scale, cleared);
    bool good = true;
    groups([&](float x) { good &= x < CUDART_INF_F; });
    return __syncthreads_and(good);
}

// Rank 0's share of a row whose list ran over: the K largest of the whole row, by passes over the row's keys.  The rest as in collect.
template <class T, bool REST, int NT, int G, int LIST, int HOT>
__device__ __noinline__ void select_row(TopList<NT, G, LIST, HOT> &sh, const T *row, int V, uint32_t K, float scale, Rest &rest) {
    constexpr int P = kPer<T>;
    const Share s = share<T>(row, V, 0, V);
    auto words = [&](auto f) {
        for (int w = threadIdx.x; w < s.words; w += NT) {
            float x[P];
            unpack(load_word(row, s, w), x);
            f(w, x);
        }
    };
    uint32_t key = 0, left = K;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int b = threadIdx.x; b < 256; b += NT) sh.count[b] = 0;
        __syncthreads();
        words([&](int, const float (&x)[P]) {
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const uint32_t k = key_of(x[e]);
                if (k > kKeyMasked && ((uint64_t)(k ^ key) >> (shift + 8)) == 0) atomicAdd(&sh.count[k >> shift & 255], 1u);
            }
        });
        __syncthreads();
        if (threadIdx.x == 0) {
            uint32_t above = 0;
            int b = 255;
            while (b > 0 && above + sh.count[b] < left) above += sh.count[b--];
            sh.scan[0] = (uint32_t)b;
            sh.scan[1] = left - above;
        }
        __syncthreads();
        key |= sh.scan[0] << shift;
        left = sh.scan[1];
    }
    // everything above the key, and of the equal ones the first `left`
    if (threadIdx.x == 0) sh.listed = 0;
    rest = Rest();
    uint32_t equal = 0;
    for (int w0 = 0; w0 < s.words; w0 += NT) {
        const int w = w0 + threadIdx.x;
        float x[P];
        unpack(w < s.words ? load_word(row, s, w) : masked_word<T>(), x);
        uint32_t mine = 0;
#pragma unroll
        for (int e = 0; e < P; ++e) mine += key_of(x[e]) == key;
        const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
        uint32_t up = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(kFull, up, o);
            if (lane >= o) up += y;
        }
        __syncthreads();
        if (lane == 31) sh.scan[warp] = up;
        __syncthreads();
        uint32_t at = equal + up - mine;
        for (int v = 0; v < NT / 32; ++v) {
            if (v < warp) at += sh.scan[v];
            equal += sh.scan[v];
        }
#pragma unroll
        for (int e = 0; e < P; ++e) {
            const uint32_t k = key_of(x[e]);
            if (k <= kKeyMasked) continue;
            if (k > key || (k == key && at++ < left)) sh.list[next_place(&sh.listed)] = entry_of(x[e], s.first + w * P - s.mis + e);
            else if (REST) rest.add(x[e], scale);
        }
    }
    __syncthreads();
}

}  // namespace rows
}  // namespace dsbd
