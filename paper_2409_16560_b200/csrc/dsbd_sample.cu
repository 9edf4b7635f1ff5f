// Draws from rows of logits with each row's own temperature, top-k, top-p and min-p, and the largest logits of rows.
//
// A row belongs to a cluster of 1 to 8 CTAs, which brings it into shared memory once; every later step reads it there.
//
// Cuts.  Temperature, top-k, top-p and min-p all keep a prefix of the tokens in falling order of (logit, -token), so a row's cuts are one
// pair (key, token): kept is what lies at or above it.
//   up to kTop tokens: each thread has the largest of its words; the k-th largest of those maxima (by bins) is at or below the
//     k-th largest logit, and little more than k tokens reach it.  They go to a list in one CTA, which sorts it.
//   otherwise, or where more tokens tie than the list holds: a histogram of 512 bins over the cluster, linear in the logit first,
//     then in the bits of the keys of the bin that the cut is in, until that is one key; equal keys go by token.  Masses are
//     whole numbers (2^62 / V' of the largest token's mass, V' the power of two from V on), so sums do not depend on their order.
// The draw is the first kept token in the tokens' order whose cumulative mass exceeds u times the whole.  Masses and sums are in 64
// bits: a token changes when a sum moves across it, and a long-tailed row has cells narrower than the rounding of sums in 32 bits.
#include "dsbd_top.cuh"

namespace dsbd {
namespace rows {
namespace {

static_assert(kBins == kThreads, "a thread for each bin");
constexpr int kTop = DSBD_MAX_TOP;                 // tokens that a cut by list keeps, at most
constexpr int kList = 2 * kTop;                    // entries of the list

struct SampleArgs {
    const void *logits;
    int64_t stride;
    int rows, V, draws, ctas, per;
    float temperature, top_p, min_p;
    int top_k;
    const float *temperature_r, *top_p_r, *min_p_r;
    const int32_t *top_k_r;
    const float *uniform;
    int32_t *token;
    float *logp;
    int32_t *status;
};

struct Hist {
    uint32_t count[kBins], low[kBins], high[kBins];
};

struct Note {
    double sum;
    float high, low;
    uint32_t a, b;
};

struct Shared {
    double table[64];
    Told<Note> told;
    union {
        Hist hist[2];
        double mass[kTop];                         // of the list's entries, in the CTA that sorts
    };
    uint64_t list[kList];
    Note scratch[kWarps];
    double sums[kWarps + 1];
    uint64_t scan[kWarps];
    uint64_t picked_before;
    uint32_t picked_bin, picked_count;
    uint32_t listed;
    int found;
};

struct Cut {
    uint32_t key;
    int token;
    __device__ __forceinline__ bool keeps(uint32_t k, int t) const { return k > key || (k == key && t <= token); }
};

// A row as a CTA of its cluster sees it.
template <class T>
struct Row {
    Share s;
    const float4 *mem;
    Shared &sh;
    int ctas, rank, V;
    int note_turn, hist_turn;
    float top, low;                                // the largest logit; the smallest of the threads' finite maxima
    float mine;                                    // this thread's maximum

    __device__ __forceinline__ const Note *tell_all(const Note &n) { return tell(n, sh.told, note_turn, ctas, rank); }
    template <class P>
    __device__ __forceinline__ P *of(P *p, int c) const { return ctas > 1 ? cg::this_cluster().map_shared_rank(p, c) : p; }
    // words of a warp, in the order of the tokens: warp w has [w * n, w * n + n)
    __device__ __forceinline__ int warp_words() const { return (s.words + kWarps - 1) / kWarps; }
};

__device__ __forceinline__ Note join_top(Note x, const Note &y) {
    x.high = fmaxf(x.high, y.high);
    x.low = fminf(x.low, y.low);
    x.a |= y.a;
    return x;
}

// Brings the row, finds its largest logit.  False: the row holds a NaN or +inf, or nothing above -inf (reported).
template <class T>
__device__ __forceinline__ bool bring(Row<T> &r, const T *row, float4 *mem, int32_t *status) {
    float high = -CUDART_INF_F;
    uint32_t bad = 0;
    load_share<T>(row, r.s, mem, [&](const float (&x)[kPer<T>]) {
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) {
            high = fmaxf(high, x[e]);
            bad |= !(x[e] < CUDART_INF_F);
        }
    });
    r.mine = high;
    Note n = {0.0, high, high > -CUDART_INF_F ? high : CUDART_INF_F, bad, 0};
    n = over_cta(n, join_top, r.sh.scratch);
    begun_wait(r.ctas);
    const Note *all = r.tell_all(n);
    for (int c = 0; c < r.ctas; ++c) n = join_top(n, all[c]);
    r.top = n.high;
    r.low = n.low;
    if (n.a || !(n.high > -CUDART_INF_F)) {
        if (r.rank == 0 && threadIdx.x == 0) report(status, n.a ? DSBD_DEV_BAD_LOGIT : DSBD_DEV_EXHAUSTED);
        return false;
    }
    return true;
}

// The cluster's totals of bin threadIdx.x, after a barrier behind the filling.
template <class T>
__device__ __forceinline__ uint32_t bin_count(const Row<T> &r, Hist &h) {
    uint32_t n = 0;
    for (int c = 0; c < r.ctas; ++c) n += r.of(&h, c)->count[threadIdx.x];
    return n;
}
template <class T>
__device__ __forceinline__ uint64_t bin_mass(const Row<T> &r, Hist &h) {
    uint64_t m = 0;
    for (int c = 0; c < r.ctas; ++c) {
        const Hist *o = r.of(&h, c);
        m += ((uint64_t)o->high[threadIdx.x] << 32) + o->low[threadIdx.x];
    }
    return m;
}

template <bool BY_MASS>
__device__ __forceinline__ void clear(Hist &h) {
    h.count[threadIdx.x] = 0;
    if (BY_MASS) h.low[threadIdx.x] = h.high[threadIdx.x] = 0;
    __syncthreads();
}

// Mass as a whole number.
struct Whole {
    const Mass &mass;
    double unit;
    __device__ __forceinline__ uint64_t of(float z) const {
        // (by its bits, see widen)
        const uint64_t bits = (uint64_t)__double_as_longlong(mass.of(z) * unit);
        const int up = (int)(bits >> 52) - 1075;
        const uint64_t digits = (bits & 0xfffffffffffffull) | 0x10000000000000ull;
        return up >= 0 ? digits << up : up > -53 ? digits >> -up : 0;
    }
};

// The token of rank `rank` (from 0) among those of the share that `is` holds for, of all CTAs, in the tokens' order.
template <class T, class F>
__device__ int nth_token(Row<T> &r, uint32_t rank, F is) {
    Shared &sh = r.sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, n = r.warp_words();
    const int w0 = warp * n, w1 = min(w0 + n, r.s.words);
    auto word = [&](int w, uint32_t *which) {
        uint32_t bits = 0;
        if (w < w1) {
            float x[kPer<T>];
            unpack(r.mem[w], x);
            const int t = r.s.first + w * kPer<T> - r.s.mis;
#pragma unroll
            for (int e = 0; e < kPer<T>; ++e) bits |= (uint32_t)is(key_of(x[e]), t + e) << e;
        }
        *which = bits;
        return (uint32_t)__popc(bits);
    };
    uint32_t mine = 0, bits;
    for (int w = w0 + lane; w < w1; w += 32) mine += word(w, &bits);
    mine = __reduce_add_sync(kFull, mine);
    __syncthreads();
    if (lane == 0) sh.scan[warp] = mine;
    __syncthreads();
    uint32_t base = 0, total = 0;
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) base += (uint32_t)sh.scan[w];
        total += (uint32_t)sh.scan[w];
    }
    const Note *all = r.tell_all({0.0, 0.f, 0.f, total, 0});
    for (int c = 0; c < r.rank; ++c) base += all[c].a;
    if (rank >= base && rank - base < mine) {
        uint32_t left = rank - base;
        for (int w = w0; w < w1; w += 32) {
            const uint32_t here = word(w + lane, &bits);
            uint32_t up = here;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t x = __shfl_up_sync(kFull, up, o);
                if (lane >= o) up += x;
            }
            const uint32_t sum = __shfl_sync(kFull, up, 31);
            if (left < sum) {
                if (left < up && left >= up - here) {
                    for (uint32_t skip = left - (up - here); skip > 0; --skip) bits &= bits - 1;
                    const int t = r.s.first + (w + lane) * kPer<T> - r.s.mis + __ffs(bits) - 1;
                    for (int c = 0; c < r.ctas; ++c) *r.of(&sh.found, c) = t;
                }
                break;
            }
            left -= sum;
        }
    }
    cluster_barrier(r.ctas);
    return sh.found;
}

// The cut within `within` that keeps the k largest tokens (BY_MASS false), or the shortest prefix of at least p of the mass.
template <bool BY_MASS, class T>
__device__ Cut cut_at(Row<T> &r, Cut within, uint32_t k, double p, const Whole &whole, float width) {
    Shared &sh = r.sh;
    const float scale = bins_over(width);
    uint64_t above = 0;
    double goal = (double)k;
    uint32_t lo = 0, hi = 0xffffffffu;
    int shift = 32;
    for (bool first = true;; first = false) {
        Hist &h = sh.hist[r.hist_turn++ & 1];
        clear<BY_MASS>(h);
        each<T>(r.s, r.mem, [&](int t, float z) {
            const uint32_t key = key_of(z);
            if (!within.keeps(key, t) || (!first && (key < lo || key > hi))) return;
            const int b = first ? bin_below(r.top, z, scale) : (int)((hi - key) >> shift);
            if (BY_MASS) {
                const uint64_t m = whole.of(z);
                if (m == 0) return;
                const uint32_t low = (uint32_t)m, was = atomicAdd(&h.low[b], low);
                const uint32_t high = (uint32_t)(m >> 32) + (was + low < low);
                if (high) atomicAdd(&h.high[b], high);
            }
            atomicAdd(&h.count[b], 1u);
        });
        cluster_barrier(r.ctas);
        const uint32_t n = bin_count(r, h);
        const uint64_t v = BY_MASS ? bin_mass(r, h) : n;
        uint64_t total;
        const uint64_t excl = before(v, &total, sh.scan);
        if (BY_MASS && first) goal = p * (double)total;
        if (!BY_MASS && first && total <= k) return within;          // (masked rows may have fewer than k)
        if (v && (double)(above + excl) < goal && (double)(above + excl + v) >= goal) {
            sh.picked_bin = threadIdx.x;
            sh.picked_count = n;
            sh.picked_before = excl;
        }
        __syncthreads();
        const uint32_t bin = sh.picked_bin, count = sh.picked_count;
        above += sh.picked_before;
        if (first) {
            // (the keys of a linear bin: by looking at them)
            uint32_t least = 0xffffffffu, most = 0;
            each<T>(r.s, r.mem, [&](int t, float z) {
                const uint32_t key = key_of(z);
                if (!within.keeps(key, t) || bin_below(r.top, z, scale) != (int)bin || (BY_MASS && whole.of(z) == 0)) return;
                least = min(least, key);
                most = max(most, key);
            });
            Note m = {0.0, 0.f, 0.f, least, most};
            auto join = [](Note x, const Note &y) { x.a = min(x.a, y.a); x.b = max(x.b, y.b); return x; };
            m = over_cta(m, join, sh.scratch);
            const Note *all = r.tell_all(m);
            for (int c = 0; c < r.ctas; ++c) m = join(m, all[c]);
            lo = m.a;
            hi = m.b;
        } else {
            hi -= bin << shift;
            if ((uint64_t)hi - lo >= 1ull << shift) lo = hi - ((1u << shift) - 1);
        }
        // everything of the bin is kept: its only token, or the last one of the k
        if (count == 1 || (!BY_MASS && above + count == k)) return lo > within.key ? Cut{lo, 0x7fffffff} : Cut{max(lo, within.key), within.token};
        if (lo == hi) {
            uint32_t keep = (uint32_t)(k - above);
            if (BY_MASS) {
                const double m = (double)whole.of(of_key(lo));
                keep = (uint32_t)fmin(fmax(ceil((goal - (double)above) / m), 1.0), (double)count);
            }
            const Cut tied = {lo, lo == within.key ? within.token : 0x7fffffff};
            if (keep >= count) return tied;
            return {lo, nth_token(r, keep - 1, [&](uint32_t key, int t) { return key == lo && t <= tied.token; })};
        }
        shift = max(0, 32 - __clz(hi - lo) - 9);
        __syncthreads();                           // (what was picked has been read)
    }
}

// The tokens at or above the k-th largest logit, as (key, ~token) in falling order, in the list of rank 0; returns their
// number there, and -1 everywhere if the list does not hold them.  k <= kTop; fewer than k where the row has fewer above -inf.
template <class T>
__device__ int list_top(Row<T> &r, int k) {
    Shared &sh = r.sh;
    const float scale = bins_over(r.top - r.low);
    Hist &h = sh.hist[r.hist_turn++ & 1];
    clear<false>(h);
    if (threadIdx.x == 0) {
        sh.listed = 0;
        sh.picked_bin = kBins - 1;
    }
    if (r.mine > -CUDART_INF_F) atomicAdd(&h.count[bin_below(r.top, r.mine, scale)], 1u);
    cluster_barrier(r.ctas);
    uint64_t total;
    const uint64_t n = bin_count(r, h), excl = before(n, &total, sh.scan);
    if (excl < (uint64_t)k && excl + n >= (uint64_t)k) sh.picked_bin = threadIdx.x;
    __syncthreads();
    const int last = (int)sh.picked_bin;
    each<T>(r.s, r.mem, [&](int t, float z) {
        if (z == -CUDART_INF_F || (last < kBins - 1 && (r.top - z) * scale >= (float)(last + 1))) return;
        const uint32_t at = atomicAdd(&sh.listed, 1u);
        if (at < (uint32_t)kList) sh.list[at] = ((uint64_t)key_of(z) << 32) | (uint32_t)~t;
    });
    __syncthreads();
    const Note *all = r.tell_all({0.0, 0.f, 0.f, sh.listed, 0});
    uint32_t sum = 0;
    for (int c = 0; c < r.ctas; ++c) sum += all[c].a;
    if (sum > (uint32_t)kList) return -1;
    if (r.rank == 0) {
        uint32_t at = all[0].a;
        for (int c = 1; c < r.ctas; ++c) {
            const uint64_t *from = r.of(&sh.list[0], c);
            for (uint32_t i = threadIdx.x; i < all[c].a; i += kThreads) sh.list[at + i] = from[i];
            at += all[c].a;
        }
    }
    cluster_barrier(r.ctas);                       // (the others' lists have been read)
    if (r.rank == 0) {
        int size = 2;
        while (size < (int)sum) size <<= 1;
        for (int i = sum + threadIdx.x; i < size; i += kThreads) sh.list[i] = 0;
        sort_down(sh.list, size);
    }
    return (int)sum;
}


// ------------------------------------------------------------------------------------ draws
struct Settings {
    float T, p, m;
    int k;
};

// A uniform number's target in a mass of `total`: below it, so that some token exceeds it.
__device__ __forceinline__ double target(float u, double total) {
    return fmin((double)u * total, __longlong_as_double(__double_as_longlong(total) - 1));
}

__device__ __forceinline__ void no_draw(const SampleArgs &a, int row, int d, int code) {
    a.token[(int64_t)row * a.draws + d] = -1;
    if (a.logp) a.logp[(int64_t)row * a.draws + d] = CUDART_NAN_F;
    if (code) report(a.status, code);
}

__device__ __forceinline__ void put_draw(const SampleArgs &a, int row, int d, int token, double logp) {
    a.token[(int64_t)row * a.draws + d] = token;
    if (a.logp) a.logp[(int64_t)row * a.draws + d] = (float)logp;
}

// Draws of a list of n entries in falling order (rank 0 alone): its cuts are prefixes.
template <class T>
__device__ void draw_listed(Row<T> &r, const SampleArgs &a, int row, const Settings &set, int n, const Mass &mass) {
    Shared &sh = r.sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    n = min(n, set.k);
    constexpr int kMine = kTop / kThreads;         // entries of a thread, side by side
    double w[kMine], total, mine = 0.0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int at = threadIdx.x * kMine + i;
        w[i] = at < n ? mass.of(logit_of(sh.list[at])) : 0.0;
        mine += w[i];
    }
    double upto = before(mine, &total, sh.sums);
    uint32_t out = 0x7fffffffu;                    // the first entry that is cut off
#pragma unroll
    for (int i = kMine - 1; i >= 0; --i) {
        double b = upto;
        for (int j = 0; j < i; ++j) b += w[j];
        const int at = threadIdx.x * kMine + i;
        if (at < n && ((set.p < 1.f && !(b < (double)set.p * total)) || !(w[i] >= (double)set.m))) out = at;
    }
    n = (int)min((uint32_t)n, over_cta(out, [](uint32_t x, uint32_t y) { return min(x, y); }, reinterpret_cast<uint32_t *>(sh.scratch)));
    // the kept ones in the tokens' order: (~token, place) falling
    uint64_t e[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int at = threadIdx.x * kMine + i;
        e[i] = at < n ? sh.list[at] : 0;
    }
    __syncthreads();
    int size = 2;
    while (size < n) size <<= 1;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int at = threadIdx.x * kMine + i;
        if (at < size) sh.list[at] = at < n ? (e[i] << 32) | (e[i] >> 32) : 0;
    }
    sort_down(sh.list, size);
    mine = 0.0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int at = threadIdx.x * kMine + i;
        w[i] = at < n ? mass.of(of_key((uint32_t)sh.list[at])) : 0.0;
        mine += w[i];
    }
    upto = before(mine, &total, sh.sums);
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        upto += w[i];
        const int at = threadIdx.x * kMine + i;
        if (at < n) sh.mass[at] = upto;
    }
    __syncthreads();
    total = sh.mass[n - 1];
    for (int d = warp; d < a.draws; d += kWarps) {
        const float u = a.uniform[(int64_t)row * a.draws + d];
        if (!(u >= 0.f && u <= 1.f)) {
            if (lane == 0) no_draw(a, row, d, DSBD_DEV_BAD_PARAM);
            continue;
        }
        const double t = target(u, total);
        int at = 0;
        for (int i = lane; i < n; i += 32) at += sh.mass[i] <= t;
        at = min((int)__reduce_add_sync(kFull, (unsigned)at), n - 1);
        if (lane == 0) {
            const uint64_t x = sh.list[at];
            put_draw(a, row, d, (int)~(uint32_t)(x >> 32),
                     ((double)of_key((uint32_t)x) - (double)r.top) / (double)set.T - log(total));
        }
    }
}

// Draws of all tokens that the cut keeps and that have at least m of the largest one's mass, each CTA its share's.
template <class T>
__device__ void draw_shared(Row<T> &r, const SampleArgs &a, int row, const Settings &set, Cut cut, const Mass &mass) {
    Shared &sh = r.sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, n = r.warp_words();
    const int w0 = warp * n, w1 = min(w0 + n, r.s.words);
    const double least = (double)set.m, top = (double)r.top;
    const float z_cut = of_key(cut.key);
    auto word = [&](int w, double (&m)[kPer<T>]) {
        float x[kPer<T>];
        unpack(r.mem[w], x);
        const int t = r.s.first + w * kPer<T> - r.s.mis;
        double sum = 0.0;
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) {
            m[e] = x[e] > z_cut || (x[e] == z_cut && t + e <= cut.token) ? mass.of(x[e]) : 0.0;
            if (!(m[e] >= least)) m[e] = 0.0;
            sum += m[e];
        }
        return sum;
    };
    double mine = 0.0, m[kPer<T>];
    for (int w = w0 + lane; w < w1; w += 32) mine += word(w, m);
    mine = warp_sum(mine);
    __syncthreads();
    if (lane == 0) sh.sums[warp] = mine;
    __syncthreads();
    // where each warp's masses begin in its CTA; sums of the same numbers in the same order wherever they are needed
    double begin = 0.0, end = 0.0;
    for (int w = 0; w < kWarps; ++w) {
        if (w == warp) begin = end;
        end += sh.sums[w];
    }
    const Note *all = r.tell_all({end, 0.f, 0.f, 0, 0});
    double base = 0.0, total = 0.0;
    for (int c = 0; c < r.ctas; ++c) {
        if (c == r.rank) base = total;
        total += all[c].sum;
    }
    const double lo = base + begin, hi = base + (begin + mine);
    for (int d = 0; d < a.draws; ++d) {
        const float u = a.uniform[(int64_t)row * a.draws + d];
        if (!(u >= 0.f && u <= 1.f)) {
            if (r.rank == 0 && threadIdx.x == 0) no_draw(a, row, d, DSBD_DEV_BAD_PARAM);
            continue;
        }
        const double t = target(u, total);
        if (!(lo <= t && t < hi)) continue;
        double done = lo;
        int token = -1;
        float z = 0.f;
        for (int w = w0; w < w1; w += 32) {
            const double here = w + lane < w1 ? word(w + lane, m) : 0.0;
            double up = here;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double x = __shfl_up_sync(kFull, up, o);
                if (lane >= o) up += x;
            }
            // the first lane that goes beyond t; where rounding lets none, the last one with a mass
            const unsigned beyond = __ballot_sync(kFull, done + up > t && here > 0.0);
            const unsigned some = __ballot_sync(kFull, here > 0.0);
            const int who = beyond ? __ffs(beyond) - 1 : 31 - __clz(some);
            if (some && lane == who) {
                double c = done + (up - here);
                float x[kPer<T>];
                unpack(r.mem[w + lane], x);
                const int first = r.s.first + (w + lane) * kPer<T> - r.s.mis;
                for (int e = 0; e < kPer<T>; ++e) {
                    if (m[e] == 0.0) continue;
                    token = first + e;
                    z = x[e];
                    c += m[e];
                    if (c > t) break;
                }
            }
            if (some) {
                token = __shfl_sync(kFull, token, who);
                z = __shfl_sync(kFull, z, who);
            }
            if (beyond) break;
            done += __shfl_sync(kFull, up, 31);
        }
        if (lane == 0) put_draw(a, row, d, token, ((double)z - top) / (double)set.T - log(total));
    }
}

template <class T>
__global__ void __launch_bounds__(kThreads) k_sample(SampleArgs a) {
    extern __shared__ float4 mem[];
    __shared__ Shared sh;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    begun_arrive(a.ctas);
    const int row = blockIdx.x / a.ctas;
    Settings set = {a.temperature, a.top_p, a.min_p, a.top_k};
    if (a.temperature_r) set.T = a.temperature_r[row];
    if (a.top_p_r) set.p = a.top_p_r[row];
    if (a.min_p_r) set.m = a.min_p_r[row];
    if (a.top_k_r) set.k = a.top_k_r[row];
    const int rank = blockIdx.x - row * a.ctas;
    const bool valid = set.T >= 0.f && set.T < CUDART_INF_F && set.p > 0.f && set.m >= 0.f && set.m <= 1.f;
    const T *at = static_cast<const T *>(a.logits) + (int64_t)row * a.stride;
    Row<T> r = {share<T>(at, a.V, rank, a.per), mem, sh, a.ctas, rank, a.V, 0, 0, 0.f, 0.f, 0.f};
    Mass::fill(sh.table);
    if (!valid) begun_wait(a.ctas);
    if (!valid || !bring<T>(r, at, mem, a.status)) {
        if (rank == 0)
            for (int d = threadIdx.x; d < a.draws; d += kThreads) no_draw(a, row, d, valid ? 0 : DSBD_DEV_BAD_PARAM);
        return;
    }
    if (set.T == 0.f) {
        uint32_t first = 0x7fffffffu;
        each<T>(r.s, r.mem, [&](int t, float z) { if (z == r.top) first = min(first, (uint32_t)t); });
        auto least = [](uint32_t x, uint32_t y) { return min(x, y); };
        first = over_cta(first, least, reinterpret_cast<uint32_t *>(sh.scratch));
        const Note *all = r.tell_all({0.0, 0.f, 0.f, first, 0});
        for (int c = 0; c < a.ctas; ++c) first = min(first, all[c].a);
        if (rank == 0)
            for (int d = threadIdx.x; d < a.draws; d += kThreads) {
                const float u = a.uniform[(int64_t)row * a.draws + d];
                if (u >= 0.f && u <= 1.f) put_draw(a, row, d, (int)first, 0.0);
                else no_draw(a, row, d, DSBD_DEV_BAD_PARAM);
            }
        return;
    }
    const Mass mass(set.T, r.top, sh.table);
    Cut cut = {kKeyMasked, -1};                    // everything above -inf
    const bool by_rank = set.k > 0 && set.k < a.V;
    if (by_rank && set.k <= kTop) {
        const int n = list_top(r, set.k);
        if (n >= 0) {
            if (rank == 0) draw_listed(r, a, row, set, n, mass);
            return;
        }
    }
    const Whole whole = {mass, (double)(1ull << (30 + __clz(a.V - 1 | 1)))};
    if (by_rank) cut = cut_at<false>(r, cut, (uint32_t)set.k, 0.0, whole, 2.f * (r.top - r.low));
    if (set.p < 1.f) cut = cut_at<true>(r, cut, 0, (double)set.p, whole, 64.f * 0.6931472f * set.T);
    draw_shared(r, a, row, set, cut, mass);
}

}  // namespace
}  // namespace rows
}  // namespace dsbd

using namespace dsbd::rows;

extern "C" int dsbd_sample_rows(const dsbd_rows_t *rows, const dsbd_sample_params_t *p, const float *uniform, int32_t *token,
                                float *logp, int32_t *status, dsbd_stream_t stream) {
    int rc = check_rows(rows);
    if (rc) return rc;
    if (!p || p->draws < 0 || !status) return DSBD_ERR_INVALID_ARG;
    if (!p->temperature_r && !(p->temperature >= 0.f && p->temperature <= FLT_MAX)) return DSBD_ERR_INVALID_ARG;
    if (!p->top_p_r && !(p->top_p > 0.f)) return DSBD_ERR_INVALID_ARG;
    if (!p->min_p_r && !(p->min_p >= 0.f && p->min_p <= 1.f)) return DSBD_ERR_INVALID_ARG;
    if (rows->rows == 0 || p->draws == 0) return DSBD_OK;
    if (!rows->logits || !uniform || !token) return DSBD_ERR_INVALID_ARG;
    const Plan plan = plan_for(rows);
    SampleArgs a = {};
    a.logits = rows->logits; a.stride = rows->row_stride; a.rows = rows->rows; a.V = rows->V; a.draws = p->draws;
    a.ctas = plan.ctas; a.per = plan.per;
    a.temperature = p->temperature; a.top_p = p->top_p; a.min_p = p->min_p; a.top_k = p->top_k;
    a.temperature_r = p->temperature_r; a.top_p_r = p->top_p_r; a.min_p_r = p->min_p_r; a.top_k_r = p->top_k_r;
    a.uniform = uniform; a.token = token; a.logp = logp; a.status = status;
    return rows->dtype == DSBD_DTYPE_F32 ? launch(k_sample<float>, rows->rows, plan, 0, a, stream)
                                         : launch(k_sample<__nv_bfloat16>, rows->rows, plan, 0, a, stream);
}
