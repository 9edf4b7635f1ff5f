// Rows of logits in the shared memory of a cluster: what the draws, the largest logits and the distillation share.
#pragma once

#include <cfloat>
#include <climits>

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <math_constants.h>

#include "dsbd_common.cuh"

namespace dsbd {
namespace rows {

namespace cg = cooperative_groups;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCtas = 8;                        // the largest portable cluster

// ---- elements ------------------------------------------------------------------------------
template <class T> constexpr int kPer = 16 / (int)sizeof(T);     // elements of a 16-byte word

__device__ __forceinline__ float value_of(float x) { return x; }
__device__ __forceinline__ float value_of(__nv_bfloat16 x) { return __bfloat162float(x); }

__device__ __forceinline__ void unpack(const float4 &w, float (&x)[4]) { x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w; }
__device__ __forceinline__ void unpack(const float4 &w, float (&x)[8]) {
    const uint32_t u[4] = {__float_as_uint(w.x), __float_as_uint(w.y), __float_as_uint(w.z), __float_as_uint(w.w)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ float4 pack(const float (&x)[4]) { return make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ float4 pack(const float (&x)[8]) {
    float4 w;
    float *o = &w.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 two = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        o[i] = __uint_as_float(*reinterpret_cast<const uint32_t *>(&two));
    }
    return w;
}

// Order of floats as order of unsigned numbers, -0 as +0.
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t u = __float_as_uint(z + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) {
    return __uint_as_float(k ^ ((uint32_t)((int32_t)~k >> 31) | 0x80000000u));
}
constexpr uint32_t kKeyMasked = 0x007fffffu;       // key_of(-inf)

// ---- a row's share of a CTA --------------------------------------------------------------------
// CTA c of the cluster holds the tokens [first, first + count), token t at position mis + t - first of its shared memory, so that
// 16-byte words lie in shared memory as they do in the row, whatever the row's alignment; what a first or last word holds besides
// is -inf.  Shares are multiples of 16 elements, so all of a row's CTAs have the same mis.
struct Share {
    int first, count, mis, words;
};

inline int share_of(int V, int ctas) { return ((V + ctas - 1) / ctas + 15) / 16 * 16; }

template <class T>
__device__ __forceinline__ Share share(const T *row, int V, int rank, int per) {
    Share s;
    s.first = min(rank * per, V);
    s.count = min(per, V - s.first);
    s.mis = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    s.words = s.count > 0 ? (s.mis + s.count + kPer<T> - 1) / kPer<T> : 0;
    return s;
}

// Word w of the share, from the row: the elements that are the share's, -inf for the others.
template <class T>
__device__ __forceinline__ float4 load_word(const T *row, const Share &s, int w) {
    constexpr int P = kPer<T>;
    const int at = w * P - s.mis;                  // of its first element in the share
    const T *p = row + s.first + at;
    if (at >= 0 && at + P <= s.count) return ld_stream(reinterpret_cast<const float4 *>(p));
    float x[P];
#pragma unroll
    for (int e = 0; e < P; ++e) x[e] = at + e >= 0 && at + e < s.count ? value_of(p[e]) : -CUDART_INF_F;
    return pack(x);
}

template <class T>
__device__ __forceinline__ float4 masked_word() {
    float x[kPer<T>];
#pragma unroll
    for (int e = 0; e < kPer<T>; ++e) x[e] = -CUDART_INF_F;
    return pack(x);
}

// 16-byte words of a thread in a batch: 32 elements.
template <class T> constexpr int kDeep = 32 / kPer<T>;
// Word u of this thread in the batch from word w0 on: a warp's words of a batch lie side by side.
template <int D>
__device__ __forceinline__ int batch_word(int w0, int u) {
    return w0 + (threadIdx.x / 32 * D + u) * 32 + (threadIdx.x & 31);
}

template <class T, int NT>
__device__ __forceinline__ void load_batch(float4 (&raw)[kDeep<T>], const T *row, const Share &s, int w0) {
    constexpr int D = kDeep<T>;
    if (w0 > 0 && w0 + D * NT < s.words) {
        const float4 *p = reinterpret_cast<const float4 *>(row + s.first - s.mis) + batch_word<D>(w0, 0);
#pragma unroll
        for (int u = 0; u < D; ++u) raw[u] = ld_stream(p + u * 32);
    } else {
#pragma unroll
        for (int u = 0; u < D; ++u) raw[u] = batch_word<D>(w0, u) < s.words ? load_word(row, s, batch_word<D>(w0, u)) : masked_word<T>();
    }
}

// The share into shared memory, 8 words a thread in flight, each also to f(elements) of the thread that brought it.
template <class T, class F>
__device__ __forceinline__ void load_share(const T *row, const Share &s, float4 *mem, F f) {
    constexpr int kDeep = 8;
    for (int w0 = threadIdx.x; w0 < s.words; w0 += kDeep * kThreads) {
        float4 raw[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
            if (w0 + u * kThreads < s.words) raw[u] = load_word(row, s, w0 + u * kThreads);
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
            if (w0 + u * kThreads < s.words) {
                mem[w0 + u * kThreads] = raw[u];
                float x[kPer<T>];
                unpack(raw[u], x);
                f(x);
            }
    }
}

// f(token, z) for this thread's elements of the share, in the words that it brought.
template <class T, class F>
__device__ __forceinline__ void each(const Share &s, const float4 *mem, F f) {
#pragma unroll 2
    for (int w = threadIdx.x; w < s.words; w += kThreads) {
        float x[kPer<T>];
        unpack(mem[w], x);
        const int t = s.first + w * kPer<T> - s.mis;
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) f(t + e, x[e]);
    }
}

// ---- over a CTA, over a cluster -----------------------------------------------------------------
template <class P>
__device__ __forceinline__ P shuffle_xor(P v, int o) {
    static_assert(sizeof(P) % 4 == 0, "");
    uint32_t u[sizeof(P) / 4];
    memcpy(u, &v, sizeof(P));
#pragma unroll
    for (unsigned i = 0; i < sizeof(P) / 4; ++i) u[i] = __shfl_xor_sync(kFull, u[i], o);
    memcpy(&v, u, sizeof(P));
    return v;
}

// All threads' v, joined, to all threads.  The joining order is fixed.  scratch: kWarps entries that nobody uses.
template <int NT = kThreads, class P, class F>
__device__ __forceinline__ P over_cta(P v, F join, P *scratch) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = join(v, shuffle_xor(v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x / 32] = v;
    __syncthreads();
    v = scratch[threadIdx.x & (NT / 32 - 1)];
#pragma unroll
    for (int o = NT / 64; o > 0; o >>= 1) v = join(v, shuffle_xor(v, o));
    return v;
}

// A place behind *n in shared memory.  (atomicAdd of a constant becomes a vote of the warp's active lanes and a leader's addition, three times the
// instructions where one lane comes, as nearly always here.)
__device__ __forceinline__ uint32_t next_place(uint32_t *n) {
    uint32_t was;
    asm volatile("atom.shared.add.u32 %0, [%1], 1;" : "=r"(was) : "r"((uint32_t)__cvta_generic_to_shared(n)) : "memory");
    return was;
}

__device__ __forceinline__ double add(double x, double y) { return x + y; }

// Over a warp without shuffles, which wait in one queue with the loads and stores of all of an SM's warps: 250 cycles each beside CTAs that
// stream.  Largest of numbers that are not NaN:
__device__ __forceinline__ float warp_most(float x) { return of_key(__reduce_max_sync(kFull, key_of(x))); }

// Sum of numbers in [0, 512), in steps of 2^-39 (so in no order); NaN if one is.
__device__ __forceinline__ double warp_total(float x) {
    const uint32_t high = (uint32_t)(x * 0x1p15f), low = (uint32_t)(fmaf((float)high, -0x1p-15f, x) * 0x1p39f);
    const double sum = (double)__reduce_add_sync(kFull, high) * 0x1p-15 + (double)__reduce_add_sync(kFull, low) * 0x1p-39;
    return __any_sync(kFull, x != x) ? (double)CUDART_NAN_F : sum;
}
// The same of [0, 16), in steps of 2^-44.
__device__ __forceinline__ double warp_total(double x) {
    const uint32_t high = (uint32_t)(x * 0x1p20), low = (uint32_t)(fma((double)high, -0x1p-20, x) * 0x1p44);
    const double sum = (double)__reduce_add_sync(kFull, high) * 0x1p-20 + (double)__reduce_add_sync(kFull, low) * 0x1p-44;
    return __any_sync(kFull, x != x) ? (double)CUDART_NAN_F : sum;
}

// 1 / x by a step of Newton's from the reciprocal in 32 bits: 2^-46 off.
__device__ __forceinline__ double inverse_of(double x) {
    const double r = (double)__frcp_rn((float)x);
    return r * fma(-x, r, 2.0);
}

// Words that the CTAs of a cluster tell one another.  Two sets, in turn: whoever writes a set for the second time has passed
// the barrier that its readers reached after reading it.
template <class P>
struct Told {
    P of[2][kMaxCtas];
};

__device__ __forceinline__ void cluster_barrier(int ctas) {
    if (ctas > 1) cg::this_cluster().sync();
    else __syncthreads();
}

// Before a CTA writes to another's shared memory, that one must have begun: arrive early, wait late.
__device__ __forceinline__ void begun_arrive(int ctas) {
    if (ctas > 1) cg::this_cluster().barrier_arrive();
}
__device__ __forceinline__ void begun_wait(int ctas) {
    if (ctas > 1) cg::this_cluster().barrier_wait();
}

// v, the same in all threads of a CTA, to all CTAs; returns the cluster's, by rank.
template <class P>
__device__ __forceinline__ const P *tell(const P &v, Told<P> &told, int &turn, int ctas, int rank) {
    P *mine = told.of[turn & 1];
    ++turn;
    if (ctas == 1) {
        if (threadIdx.x == 0) mine[0] = v;
    } else if ((int)threadIdx.x < ctas) {
        *cg::this_cluster().map_shared_rank(mine + rank, threadIdx.x) = v;
    }
    cluster_barrier(ctas);
    return mine;
}

// ---- exponentials in 32 bits, and in 64 --------------------------------------------------------------
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float max_nan(float x, float y) {
    float z;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}

// Two numbers in one instruction.
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
    float2 z;
    asm("{.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(z.x), "=f"(z.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
    return z;
}
__device__ __forceinline__ float2 mul2(float2 x, float2 y) {
    float2 z;
    asm("{.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(z.x), "=f"(z.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
    return z;
}
// 2^((x - top) scale) of two.
__device__ __forceinline__ float2 exp2_two(float x, float y, float top, float scale) {
    const float2 a = mul2(add2({x, y}, {-top, -top}), {scale, scale});
    return {exp2_fast(a.x), exp2_fast(a.y)};
}

// What a sum of exponentials relative to `from` is worth relative to `to`, the larger one (both may be -inf); scale: log2(e) / T.
__device__ __forceinline__ double rescale(float from, float to, double scale) {
    return from == to ? 1.0 : exp2(((double)from - (double)to) * scale);
}

// A sum of exponentials relative to the largest logit in it.
struct Sum {
    float high;
    double sum;
    __device__ __forceinline__ void add(const Sum &o, double scale) {
        const float top = fmaxf(high, o.high);
        sum = sum * rescale(high, top, scale) + o.sum * rescale(o.high, top, scale);
        high = top;
    }
};

// A sum of exponentials as one thread has it, relative to the largest logit in it.
struct Rest {
    float high = -INFINITY, sum = 0.f;
    __device__ __forceinline__ void raise(float to, float scale) {
        if (to > high) {
            sum *= exp2_fast((high - to) * scale);
            high = to;
        }
    }
    __device__ __forceinline__ void add(float z, float scale) {
        raise(z, scale);
        sum += z == -CUDART_INF_F ? 0.f : exp2_fast((z - high) * scale);
    }
    // a batch of words of which top is the largest element
    template <class T>
    __device__ __forceinline__ void add_words(const float4 (&raw)[kDeep<T>], float top, float scale) {
        raise(top, scale);
        const float from = high == -CUDART_INF_F ? 0.f : high;
        float2 s[2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
        for (int u = 0; u < kDeep<T>; ++u) {
            float x[kPer<T>];
            unpack(raw[u], x);
#pragma unroll
            for (int e = 0; e < kPer<T>; e += 2) s[u & 1] = add2(s[u & 1], exp2_two(x[e], x[e + 1], from, scale));
        }
        s[0] = add2(s[0], s[1]);
        sum += s[0].x + s[0].y;
    }
};

// exp((z - top) / T) in 64 bits: 2^(k / 64) from a table of 64, times a Taylor polynomial of 2^f for the rest, |f| <= 1 / 128: the
// table-driven scheme of P. T. P. Tang, ACM TOMS 15 (1989).  The degree 4 leaves (ln 2 / 128)^5 / 120 = 4e-14 of the value.
// Exactly 1 for the largest logit, and the same for equal ones.
struct Mass {
    double scale;                                  // 64 log2(e) / T
    double reach;                                  // 693 T: logits further below have less than 2^-999, and count as 0
    double top;
    float least;
    const double *table;                           // 64 entries in shared memory

    static __device__ __forceinline__ void fill(double *table) {
        if (threadIdx.x < 64) table[threadIdx.x] = exp2((double)threadIdx.x / 64.0);
    }
    __device__ __forceinline__ Mass(float T, float top, const double *table)
        : scale(64.0 * 1.4426950408889634 / (double)T), reach(693.0 * (double)T), table(table) {
        relative_to(top);
    }
    __device__ __forceinline__ void relative_to(float top) {
        this->top = (double)top;
        // (nothing: 0; -inf at no temperature.  Rounded up: where logits lie further apart than reach, the number below it would let one through
        // whose exponent leaves the range)
        least = top > -CUDART_INF_F ? fmaxf(__double2float_ru((double)top - reach), -FLT_MAX) : CUDART_INF_F;
    }
    // z <= top, not -inf
    __device__ __forceinline__ double at(float z) const {
        const double d = (double)z - top;
        const double magic = 6755399441055744.0;   // 1.5 * 2^52: adding it rounds to whole numbers
        const double t = fma(d, scale, magic);
        const int k = __double2loint(t);
        const double f = fma(d, scale, magic - t);
        constexpr double kUnit = 0.6931471805599453 / 64.0;
        double r = kUnit * kUnit * kUnit * kUnit / 24.0;
        r = fma(r, f, kUnit * kUnit * kUnit / 6.0);
        r = fma(r, f, kUnit * kUnit / 2.0);
        r = fma(r, f, kUnit);
        r = fma(r, f, 1.0);
        r *= table[k & 63];
        return __hiloint2double(__double2hiint(r) + ((k & ~63) << 14), __double2loint(r));
    }
    // 0 for -inf (no branch: the steps of several logits take turns)
    __device__ __forceinline__ double of(float z) const {
        const double m = at(fmaxf(z, least));
        return z >= least ? m : 0.0;
    }
    // of a word's elements together
    template <int P>
    __device__ __forceinline__ double of_word(const float (&x)[P]) const {
        double m[P];
#pragma unroll
        for (int e = 0; e < P; ++e) m[e] = of(x[e]);
#pragma unroll
        for (int d = P / 2; d > 0; d /= 2)
#pragma unroll
            for (int e = 0; e < d; ++e) m[e] += m[e + d];
        return m[0];
    }
};

// ---- sorting and scanning in a CTA ---------------------------------------------------------------
// Bitonic sort of n numbers (a power of two), largest first.
template <int NT = kThreads>
__device__ __forceinline__ void sort_down(uint64_t *list, int n) {
    for (int size = 2; size <= n; size <<= 1)
        for (int step = size >> 1; step > 0; step >>= 1) {
            __syncthreads();
            for (int i = threadIdx.x; i < n / 2; i += NT) {
                const int a = 2 * i - (i & (step - 1)), b = a + step;
                const uint64_t x = list[a], y = list[b];
                if ((x < y) == ((a & size) == 0)) { list[a] = y; list[b] = x; }
            }
        }
    __syncthreads();
}

// n numbers, largest first, by their bins (an order of its own: bin(x) falls nowhere as x falls), and in a bin by counting.  tmp: n numbers.  count:
// BINS numbers, scan: one for each warp.  Where a bin has many, by sort_down (list has room for a power of two then).
// A step of a sort in shared memory takes 500 cycles, 66 steps for 2048 numbers; this takes about 4000 in all.
template <int NT, int BINS, class F>
__device__ __forceinline__ void order_down(uint64_t *list, uint64_t *tmp, int n, uint32_t *count, uint32_t *scan, F bin) {
    static_assert(BINS % NT == 0, "");
    constexpr int kEach = BINS / NT;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i) count[threadIdx.x + i * NT] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) atomicAdd(&count[bin(list[i])], 1u);
    __syncthreads();
    uint32_t c[kEach], sum = 0, most = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        c[i] = count[threadIdx.x * kEach + i];
        sum += c[i];
        most = max(most, c[i]);
    }
    uint32_t up = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(kFull, up, o);
        if (lane >= o) up += x;
    }
    if (lane == 31) scan[warp] = up;
    if (__syncthreads_or(most > 48)) {
        int size = 2;
        while (size < n) size <<= 1;
        for (int i = n + threadIdx.x; i < size; i += NT) list[i] = 0;
        sort_down<NT>(list, size);
        return;
    }
    uint32_t at = up - sum;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) at += w < warp ? scan[w] : 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        count[threadIdx.x * kEach + i] = at;
        at += c[i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) {
        const uint64_t x = list[i];
        tmp[atomicAdd(&count[bin(x)], 1u)] = x;
    }
    __syncthreads();
    // (count: where each bin ends)
    for (int i = threadIdx.x; i < n; i += NT) {
        const uint64_t x = tmp[i];
        const int b = bin(x);
        const uint32_t begin = b ? count[b - 1] : 0, end = count[b];
        uint32_t rank = begin;
        for (uint32_t k = begin; k < end; ++k) rank += tmp[k] > x;
        list[rank] = x;
    }
    __syncthreads();
}

template <class P>
__device__ __forceinline__ P shuffle_up(P v, int o) {
    uint32_t u[sizeof(P) / 4];
    memcpy(u, &v, sizeof(P));
#pragma unroll
    for (unsigned i = 0; i < sizeof(P) / 4; ++i) u[i] = __shfl_up_sync(kFull, u[i], o);
    memcpy(&v, u, sizeof(P));
    return v;
}

// Sum of the v of the threads before this one; *total: of all.  scratch: an entry for each warp.
template <int NT = kThreads, class P>
__device__ __forceinline__ P before(P v, P *total, P *scratch) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    P up = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const P x = shuffle_up(up, o);
        if (lane >= o) up += x;
    }
    __syncthreads();
    if (lane == 31) scratch[warp] = up;
    __syncthreads();
    P base = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        const P x = scratch[w];
        if (w < warp) base += x;
        all += x;
    }
    *total = all;
    const P excl = shuffle_up(up, 1);
    return base + (lane ? excl : P(0));
}

// ---- launches ----------------------------------------------------------------------------------
inline int check_rows(const dsbd_rows_t *r) {
    if (!r || r->rows < 0 || r->V <= 0 || (r->rows > 1 && r->row_stride < r->V)) return DSBD_ERR_INVALID_ARG;
    if (r->dtype != DSBD_DTYPE_F32 && r->dtype != DSBD_DTYPE_BF16) return DSBD_ERR_UNSUPPORTED;
    const int size = r->dtype == DSBD_DTYPE_F32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(r->logits) & (size - 1)) || (int64_t)r->V * size > DSBD_MAX_ROW_BYTES) return DSBD_ERR_UNSUPPORTED;
    return r->rows > INT_MAX / kMaxCtas ? DSBD_ERR_UNSUPPORTED : DSBD_OK;
}

// Temperatures for sums in 32 bits: below, 1 / T overflows; above, a difference of two logits may overflow that is still worth something.
inline bool scales(float T) { return T >= FLT_MIN && T <= 0x1p100f; }

// CTAs of a row and their shares, in elements.
struct Plan {
    int ctas, per, words;
};

inline Plan plan_for(const dsbd_rows_t *r) {
    const int size = r->dtype == DSBD_DTYPE_F32 ? 4 : 2;
    Plan p;
    p.ctas = 1;
    while (p.ctas < kMaxCtas && (int64_t)share_of(r->V, p.ctas) * size > 64 * 1024) p.ctas *= 2;
    while (p.ctas < kMaxCtas && r->rows * (int64_t)p.ctas < 148 && (int64_t)share_of(r->V, p.ctas) * size > 16 * 1024) p.ctas *= 2;
    p.per = share_of(r->V, p.ctas);
    p.words = p.per * size / 16 + 1;
    return p;
}

// CTAs of a row for a kernel of which `slots` CTAs run at once: what takes least time, the CTAs in waves of that many, a CTA's time
// its share and what it does besides, `fixed` elements' worth.  No share below `least` elements.
inline Plan plan_waves(const dsbd_rows_t *r, int slots, int fixed, int least, int most) {
    Plan p = {1, 0, 0};
    int64_t best = INT64_MAX;
    for (int ctas = 1; ctas <= most && (ctas == 1 || share_of(r->V, ctas) >= least); ctas *= 2) {
        const int64_t time = (r->rows * (int64_t)ctas + slots - 1) / slots * (share_of(r->V, ctas) + fixed);
        if (time >= best) continue;
        best = time;
        p.ctas = ctas;
    }
    p.per = share_of(r->V, p.ctas);
    return p;
}

// 16-byte words of the longest share, of a row of DSBD_MAX_ROW_BYTES in kMaxCtas CTAs.
constexpr int kLongestShare = DSBD_MAX_ROW_BYTES / kMaxCtas / 16 + 1;

// MOST: the most that any call asks of the kernel's dynamic shared memory.  The limit is the whole process's, so it is this for every call: between
// one thread's setting and its launch another thread may set it for a row of its own.
template <int MOST, int NT = kThreads, class Args>
int launch(void (*kernel)(Args), int rows, const Plan &p, size_t bytes, const Args &a, dsbd_stream_t stream) {
    if (bytes > (size_t)MOST ||
        (bytes > 16 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST) != cudaSuccess)) {
        cudaGetLastError();
        return DSBD_ERR_CUDA;
    }
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * p.ctas));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = reinterpret_cast<cudaStream_t>(stream);
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelEx(&cfg, kernel, a) == cudaSuccess) return DSBD_OK;
    cudaGetLastError();
    return DSBD_ERR_CUDA;
}

}  // namespace rows
}  // namespace dsbd
