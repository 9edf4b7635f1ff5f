// Draws from rows of logits with each row's own temperature, top-k, top-p and min-p.
//
// The draw is the first kept token in the tokens' order whose cumulative mass exceeds u times the whole.  Masses and sums are in 64
// bits: a token changes when a sum moves across it, and a long-tailed row has cells narrower than the rounding of sums in 32 bits.
//
// Temperature, top-k, top-p and min-p all keep a prefix of the tokens in falling order of (logit, -token).
//   k_draw: rows that need one pass.  No cut: each warp's batches of 1024 tokens leave their mass, relative to their largest logit; the
//     batch that the target falls into is read again.  Top-k up to a few hundred (and with it top-p and min-p), or the largest logit: the k
//     largest logits come to a list in one CTA, sorted, and all the rest is done there.
//   k_draw_cut: the other rows.  A cluster of 1 to 8 CTAs brings the row into shared memory once; every later step reads it there.
//     Larger top-k: the k-th largest of the words' maxima (by bins) is at or below the k-th largest
//     logit, and little more than k tokens reach it.  Top-p, min-p: a histogram of masses by bins of the logit, rounded down a little, says which
//     bins certainly hold the prefix.  These tokens go to a list in one CTA, as above; where they are too many for it, those of the bins
//     that the cut may lie in do, and all CTAs draw from their shares.
//     Where the list does not hold these either: a histogram of 512 bins over the cluster, linear in the logit first, then in the bits of the
//     keys of the bin that the cut is in, until that is one key; equal keys go by token.  Masses are then whole numbers (Whole), so sums do not
//     depend on their order.  Then the draw over all shares.
#include <algorithm>

#include "dsbd_top.cuh"

namespace dsbd {
namespace rows {
namespace {

static_assert(kBins == kThreads, "a thread for each bin");
constexpr int kList = 4096;                        // entries of the list
// Top-k that a cut by list takes, at most.  Beyond that it is longer than the list often; and in bf16 many logits are equal, which is what
// putting it in order suffers from (64 rows of 32000, top-k 1500: 40 us, by bins 34; fp32 of 128256, top-k 2000: 53, by bins 76).
template <class T>
constexpr int kTop = sizeof(T) == 4 ? 2048 : 1024;
constexpr int kNear = 256;                         // entries that are compared with one another

struct SampleArgs {
    const void *logits;
    int64_t stride;
    int V, draws, ctas, per;
    int list_most;                                 // largest top-k that k_draw takes
    int beside;                                    // k_draw_cut: k_draw has been launched just before
    int words, list_room;                          // k_draw_cut: 16-byte words of shared memory before the list, entries of the list
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
    alignas(16) Hist hist[2];
    Note scratch[kWarps];
    double sums[kWarps + 1];
    uint64_t scan[kWarps];
    uint64_t picked_goal;
    uint32_t picked_bin, picked_count;
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
    uint64_t *list;                                // of `room` entries
    int room, ctas, rank;
    int note_turn, hist_turn;
    float top, low;                                // the largest logit; the smallest of the threads' finite maxima

    // (rank 0, which needs its share no more once the list is whole)
    __device__ __forceinline__ uint64_t *tmp() const { return reinterpret_cast<uint64_t *>(const_cast<float4 *>(mem)); }
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
__device__ __forceinline__ uint64_t bin_count(const Row<T> &r, Hist &h) {
    uint64_t n = 0;
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

// Mass as a whole number, in units of 2^-more / unit of the largest one's.  unit is 2^62 / V', V' the power of two from V on, and a token in bin b of the
// 64 octaves has at most 2^-(b / 8): with more_of(b) units, masses keep 2^-41 of themselves or better down to 2^-38 of the largest, and a bin's
// sum stays below 2^62.  (Units of one size leave a tail of masses of 2^-30 few digits: V 262144, top-p 0.9999, 4 of 115309 tokens lost.)
constexpr int kMore = 38;
__device__ __forceinline__ int more_of(int bin) { return min(bin / 8, kMore); }

struct Whole {
    const Mass &mass;
    double unit;
    __device__ __forceinline__ uint64_t of(float z, int more) const {
        // (by its bits: the conversion to whole numbers of 64 bits takes a loop)
        const uint64_t bits = (uint64_t)__double_as_longlong(mass.of(z) * unit);
        const int up = (int)(bits >> 52) - 1075 + more;
        const uint64_t digits = (bits & 0xfffffffffffffull) | 0x10000000000000ull;
        return up >= 0 ? digits << up : up > -53 ? digits >> -up : 0;
    }
};

// Sums over bins of different units: up to 2^100.
struct Wide {
    uint64_t low, high;
    __device__ __forceinline__ Wide(uint64_t low = 0, uint64_t high = 0) : low(low), high(high) {}
    __device__ __forceinline__ Wide &operator+=(const Wide &o) {
        low += o.low;
        high += o.high + (low < o.low);
        return *this;
    }
    __device__ __forceinline__ Wide operator+(const Wide &o) const { return Wide(*this) += o; }
    __device__ __forceinline__ Wide operator-(const Wide &o) const { return {low - o.low, high - o.high - (low < o.low)}; }
    __device__ __forceinline__ bool operator<(const Wide &o) const { return high < o.high || (high == o.high && low < o.low); }
    // by 1 to 127
    __device__ __forceinline__ Wide up(int n) const { return n < 64 ? Wide(low << n, high << n | low >> (64 - n)) : Wide(0, low << (n - 64)); }
    __device__ __forceinline__ Wide down(int n) const { return n < 64 ? Wide(low >> n | high << (64 - n), high >> n) : Wide(high >> (n - 64), 0); }
    // x / 2^n, rounded up
    __device__ __forceinline__ Wide part(int n) const { return (*this + (Wide(1).up(n) - Wide(1))).down(n); }
};

// p of a sum, rounded up: what a prefix that has p of it reaches.  0 < p < 1.
__device__ __forceinline__ Wide goal_of(const Wide &sum, float p) {
    const uint32_t bits = __float_as_uint(p), digits = bits & 0x7fffffu;
    const uint64_t m = bits >> 23 ? digits | 0x800000u : digits;
    const int down = bits >> 23 ? 150 - (int)(bits >> 23) : 149;
    // (sum m is below 2^124)
    return down < 124 ? Wide(sum.low * m, sum.high * m + __umul64hi(sum.low, m)).part(down) : Wide(1);
}

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

// The cut within `within` that keeps the k largest tokens (BY_MASS false), or the shortest prefix of at least p of the mass (bins of 64 octaves then).
template <bool BY_MASS, class T>
__device__ Cut cut_at(Row<T> &r, Cut within, uint32_t k, float p, const Whole &whole, float width) {
    Shared &sh = r.sh;
    const float scale = bins_over(width);
    uint64_t goal = k;                             // of what is looked at: where in it the last kept token lies
    int more = 0;
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
                const uint64_t m = whole.of(z, first ? more_of(b) : more);
                if (m == 0) return;
                const uint32_t low = (uint32_t)m, was = atomicAdd(&h.low[b], low);
                const uint32_t high = (uint32_t)(m >> 32) + (was + low < low);
                if (high) atomicAdd(&h.high[b], high);
            }
            atomicAdd(&h.count[b], 1u);
        });
        cluster_barrier(r.ctas);
        const uint32_t n = (uint32_t)bin_count(r, h);
        const uint64_t v = BY_MASS ? bin_mass(r, h) : n;
        if (BY_MASS && first) {
            const int up = kMore - more_of(threadIdx.x);
            const Wide w = up ? Wide(v).up(up) : Wide(v);
            Wide total;
            static_assert(sizeof(Note) >= sizeof(Wide) && alignof(Note) >= alignof(Wide), "");
            const Wide excl = before(w, &total, reinterpret_cast<Wide *>(sh.scratch)), end = goal_of(total, p);
            if (v && excl < end && !(excl + w < end)) {
                const Wide left = end - excl;
                sh.picked_bin = threadIdx.x;
                sh.picked_count = n;
                sh.picked_goal = up ? left.part(up).low : left.low;
            }
        } else {
            uint64_t total;
            const uint64_t excl = before(v, &total, sh.scan);
            if (!BY_MASS && first && total <= k) return within;      // (masked rows may have fewer than k)
            if (v && excl < goal && excl + v >= goal) {
                sh.picked_bin = threadIdx.x;
                sh.picked_count = n;
                sh.picked_goal = goal - excl;
            }
        }
        __syncthreads();
        const uint32_t bin = sh.picked_bin, count = sh.picked_count;
        goal = sh.picked_goal;
        if (first) {
            more = more_of(bin);
            // (the keys of a linear bin: by looking at them)
            uint32_t least = 0xffffffffu, most = 0;
            each<T>(r.s, r.mem, [&](int t, float z) {
                const uint32_t key = key_of(z);
                if (!within.keeps(key, t) || bin_below(r.top, z, scale) != (int)bin || (BY_MASS && whole.of(z, more) == 0)) return;
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
        if (count == 1 || (!BY_MASS && goal == count)) return lo > within.key ? Cut{lo, 0x7fffffff} : Cut{max(lo, within.key), within.token};
        if (lo == hi) {
            uint32_t keep = (uint32_t)goal;
            if (BY_MASS) {
                const uint64_t m = whole.of(of_key(lo), more);
                keep = (uint32_t)min((goal + m - 1) / m, (uint64_t)count);
            }
            const Cut tied = {lo, lo == within.key ? within.token : 0x7fffffff};
            if (keep >= count) return tied;
            return {lo, nth_token(r, keep - 1, [&](uint32_t key, int t) { return key == lo && t <= tied.token; })};
        }
        shift = max(0, 32 - __clz(hi - lo) - 9);
        __syncthreads();                           // (what was picked has been read)
    }
}

// What bins of width 1 / scale below top hold, by logits alone (one comparison, where a bin takes a subtraction, a product and three).  `from`: at or
// above it lie all of the bins up to `last`, and what is within a rounding of them.  `above`: at or above it lie bins before `first` alone.
struct Range {
    float from, above;
    __device__ Range(float top, float scale, int first, int last) {
        const float wide = (float)(last + 1) / scale, near = (float)first / scale;
        from = last < kBins - 1 && scale > 0.f ? fmaxf(top - wide - 4.8e-7f * (fabsf(top) + wide), -FLT_MAX) : -FLT_MAX;
        above = first ? fmaxf(top - near, -FLT_MAX) + 4.8e-7f * (fabsf(top) + near) : CUDART_INF_F;
    }
};

// The tokens with logits in a range, as (key, ~token) in the tokens' order, in the list of rank 0; returns their number, and -1 if the list does
// not hold them.  *sum: a CTA's number in, all CTAs' out.
template <class T>
__device__ int list_range(Row<T> &r, const Range range, double *sum = nullptr) {
    Shared &sh = r.sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, each_warp = r.warp_words();
    const int w0 = warp * each_warp, w1 = min(w0 + each_warp, r.s.words);
    auto marks = [&](int w) {
        uint32_t which = 0;
        if (w < w1) {
            float x[kPer<T>];
            unpack(r.mem[w], x);
#pragma unroll
            for (int e = 0; e < kPer<T>; ++e) which |= (uint32_t)(x[e] >= range.from && x[e] < range.above) << e;
        }
        return which;
    };
    // how many each warp's words have, then each entry at its place in rank 0's list (entries gathered by rank 0 instead, in reads that
    // wait for one another: 6.9 us of one row of 128256 fp32, so 5.5)
    uint32_t mine = 0;
    for (int w = w0 + lane; w < w1; w += 32) mine += __popc(marks(w));
    mine = __reduce_add_sync(kFull, mine);
    __syncthreads();
    if (lane == 0) sh.scan[warp] = mine;
    __syncthreads();
    uint32_t at = 0, listed = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        at += w < warp ? (uint32_t)sh.scan[w] : 0;
        listed += (uint32_t)sh.scan[w];
    }
    const Note *all = r.tell_all({sum ? *sum : 0.0, 0.f, 0.f, listed, 0});
    uint32_t found = 0;
    if (sum) *sum = 0.0;
    for (int c = 0; c < r.ctas; ++c) {
        at += c < r.rank ? all[c].a : 0;
        found += all[c].a;
        if (sum) *sum += all[c].sum;
    }
    if (found > (uint32_t)r.room) return -1;
    uint64_t *list = r.of(r.list, 0);
    if (mine)
        for (int w = w0; w < w1; w += 32) {
            uint32_t which = marks(w + lane), up = 0, here = 0;
#pragma unroll
            for (int e = 0; e < kPer<T>; ++e) {
                const unsigned b = __ballot_sync(kFull, which >> e & 1);
                up += __popc(b & ((1u << lane) - 1));
                here += __popc(b);
            }
            for (uint32_t to = at + up; which; which &= which - 1, ++to) {
                const int i = (w + lane) * kPer<T> + __ffs(which) - 1;
                list[to] = entry_of(value_of(reinterpret_cast<const T *>(r.mem)[i]), r.s.first + i - r.s.mis);
            }
            at += here;
        }
    cluster_barrier(r.ctas);
    return (int)found;
}

// The tokens that certainly hold the shortest prefix of p of the mass (p < 1), or those of at least m of the largest one's, listed as in
// list_range; *whole: the row's mass (p < 1).  A bin's mass is summed in steps of 2^-14 of its largest, rounded down: what is found to have p of the whole
// has it, and the list is exact.  *inside: so many bins are certainly part of the prefix.
template <class T>
__device__ int list_mass(Row<T> &r, float p, float m, float T_, const Mass &mass, double *whole, float *scale_out, int *inside, int *last_out) {
    Shared &sh = r.sh;
    constexpr float kOctaves = 16.f;               // that the bins span: a prefix that reaches further is longer than the list
    const float scale = bins_over(kOctaves * 0.6931472f * T_), step = kOctaves / (float)(kBins - 1);
    int last = kBins - 1;
    if (m > 0.f) last = min(last, (int)(-log2f(m) / step) + 1);
    if (p < 1.f) {
        Hist &h = sh.hist[r.hist_turn++ & 1];
        clear<false>(h);
        double sum = 0.0;
        for (int w = threadIdx.x; w < r.s.words; w += kThreads) {
            float x[kPer<T>];
            unpack(r.mem[w], x);
            sum += mass.of_word(x);
#pragma unroll
            for (int e = 0; e < kPer<T>; ++e) {
                const float below = (r.top - x[e]) * scale;
                if (below < (float)(kBins - 1)) {
                    const int b = (int)below;
                    atomicAdd(&h.count[b], (uint32_t)(exp2_fast(((float)b - below) * step) * 16384.f));
                }
            }
        }
        sum = over_cta(sum, add, sh.sums);
        if (threadIdx.x == 0) sh.picked_bin = kBins - 1;
        const Note *all = r.tell_all({sum, 0.f, 0.f, 0, 0});
        sum = 0.0;
        for (int c = 0; c < r.ctas; ++c) sum += all[c].sum;
        *whole = sum;
        const double v = (double)((float)bin_count(r, h) * exp2_fast(-(float)threadIdx.x * step)) * (1.0 / 16384.0);
        double all_bins;
        const double upto = before(v, &all_bins, sh.sums);
        // (the bins' sums are at most 7e-5 too small)
        const double goal = (double)p * sum;
        if (upto < goal * (1.0 + 1e-4) && upto + v >= goal * (1.0 + 1e-4)) sh.picked_bin = threadIdx.x;
        // (the last bin has no masses: what lies there, and further down, is never certain)
        *inside = __syncthreads_count(threadIdx.x < kBins - 1 && (upto + v) * (1.0 + 1e-4) < goal);
        last = min(last, (int)sh.picked_bin);
    }
    *scale_out = scale;
    *last_out = last;
    return list_range(r, Range(r.top, scale, 0, last));
}

// The cut that keeps the shortest prefix of `goal`, which lies in the bins first to last, where these are few enough for the list; false
// everywhere if not.  The mass above them is summed, they are put in order.
template <class T>
__device__ bool cut_in_bins(Row<T> &r, float scale, int first, int last, double goal, const Mass &mass, Cut *cut) {
    Shared &sh = r.sh;
    double above = 0.0;
    const Range range(r.top, scale, first, last);
    for (int w = threadIdx.x; w < r.s.words; w += kThreads) {
        float x[kPer<T>];
        unpack(r.mem[w], x);
        double m[kPer<T>];
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) m[e] = mass.of(x[e]);
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) above += x[e] >= range.above ? m[e] : 0.0;
    }
    above = over_cta(above, add, sh.sums);
    const int n = list_range(r, range, &above);
    if (n <= 0 || n > r.room / 2) return false;
    Note note = {0.0, 0.f, 0.f, 0, 0};
    if (r.rank == 0) {
        // (in the list's other half, not in the share's place: every CTA still draws from its share)
        uint64_t *tmp = r.list + r.room / 2;
        const float finer = scale * ((float)kBins / (float)(last - first + 1)), top = r.top - (float)first / scale;
        order_down<kThreads, kBins>(r.list, tmp, n, sh.hist[0].count, reinterpret_cast<uint32_t *>(sh.scan),
                                    [&](uint64_t e) { return min(max(__float2int_rz((top - logit_of(e)) * finer), 0), kBins - 1); });
        double *w = reinterpret_cast<double *>(tmp), mine = 0.0, total;
#pragma unroll 4
        for (int i = threadIdx.x; i < n; i += kThreads) w[i] = mass.of(logit_of(r.list[i]));
        if (threadIdx.x == 0) sh.picked_count = (uint32_t)n;
        __syncthreads();
        const int each = (n + kThreads - 1) / kThreads | 1, begin = min((int)threadIdx.x * each, n), end = min(begin + each, n);
        for (int i = begin; i < end; ++i) mine += w[i];
        double upto = above + before(mine, &total, sh.sums);
        for (int i = begin; i < end; ++i) {
            if (!(upto < goal)) {
                atomicMin(&sh.picked_count, (uint32_t)i);
                break;
            }
            upto += w[i];
        }
        __syncthreads();
        // the last entry that is kept (none: what is above the first)
        const int kept = (int)sh.picked_count;
        const uint64_t e = r.list[max(kept - 1, 0)];
        note.a = (uint32_t)(e >> 32);
        note.b = (uint32_t)token_of(e) - (kept == 0);
    }
    const Note got = r.tell_all(note)[0];
    *cut = {got.a, (int)got.b};
    return true;
}

// The tokens at or above the k-th largest logit, listed as in list_range.  k <= kTop<T>; fewer than k where the row has fewer above -inf.
template <class T>
__device__ int list_top(Row<T> &r, int k, float *finer) {
    Shared &sh = r.sh;
    const float scale = bins_over(r.top - r.low);
    Hist &h = sh.hist[r.hist_turn++ & 1];
    clear<false>(h);
    if (threadIdx.x == 0) sh.picked_bin = kBins - 1;
    // (a maximum of each thread instead: no faster where the list holds what reaches it, and it mostly does not where the threads are not some
    // times k: 512 rows of 32000 bf16, one CTA each, top-k 600: 109 us, so 54)
    for (int w = threadIdx.x; w < r.s.words; w += kThreads) {
        float x[kPer<T>], most = -CUDART_INF_F;
        unpack(r.mem[w], x);
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) most = fmaxf(most, x[e]);
        if (most > -CUDART_INF_F) atomicAdd(&h.count[bin_below(r.top, most, scale)], 1u);
    }
    cluster_barrier(r.ctas);
    uint64_t total;
    const uint64_t n = bin_count(r, h), excl = before(n, &total, sh.scan);
    if (excl < (uint64_t)k && excl + n >= (uint64_t)k) sh.picked_bin = threadIdx.x;
    __syncthreads();
    const int last = (int)sh.picked_bin;
    *finer = scale * ((float)kBins / (float)(last + 1));
    return list_range(r, Range(r.top, scale, 0, last));
}

// ------------------------------------------------------------------------------------ draws
struct Settings {
    float T, p, m;
    int k;                                         // 0: off
};

enum Kind { kBad, kGreedy, kListed, kPlain, kCut };

__device__ __forceinline__ Kind settings_of(const SampleArgs &a, int row, Settings &set) {
    set = {a.temperature, a.top_p, a.min_p, a.top_k};
    if (a.temperature_r) set.T = a.temperature_r[row];
    if (a.top_p_r) set.p = a.top_p_r[row];
    if (a.min_p_r) set.m = a.min_p_r[row];
    if (a.top_k_r) set.k = a.top_k_r[row];
    if (set.k <= 0 || set.k >= a.V) set.k = 0;
    if (!(set.T >= 0.f && set.T < CUDART_INF_F && set.p > 0.f && set.m >= 0.f && set.m <= 1.f)) return kBad;
    return set.T == 0.f ? kGreedy : set.k ? (set.k <= a.list_most ? kListed : kCut) : set.p >= 1.f && set.m == 0.f ? kPlain : kCut;
}

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

// Draws of a list of n entries in the tokens' order by their masses w (0: not kept).  upto_of: n numbers; sums: one for each warp.
template <int NT, int MOST>
__device__ void draw_kept(const uint64_t *list, const double *w, double *upto_of, double *sums, const SampleArgs &a, int row, const Settings &set,
                          int n, float top) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    __syncthreads();
    const int each = (n + NT - 1) / NT | 1, begin = min((int)threadIdx.x * each, n), end = min(begin + each, n);
    double total, mine = 0.0;
    for (int i = begin; i < end; ++i) mine += w[i];
    double upto = before<NT>(mine, &total, sums);
    for (int i = begin; i < end; ++i) {
        upto += w[i];
        upto_of[i] = upto;
    }
    __syncthreads();
    total = upto_of[n - 1];
    const double log_total = log(total);
    for (int d = warp; d < a.draws; d += NT / 32) {
        const float u = a.uniform[(int64_t)row * a.draws + d];
        if (!(u >= 0.f && u <= 1.f)) {
            if (lane == 0) no_draw(a, row, d, DSBD_DEV_BAD_PARAM);
            continue;
        }
        const double t = target(u, total);
        // the first entry beyond t, of those kept
        int at = 0;
        for (int step = MOST / 2; step > 0; step >>= 1)
            if (at + step <= n - 1 && upto_of[at + step - 1] <= t) at += step;
        if (lane == 0) {
            int back = at;
            while (back >= 0 && w[back] == 0.0) --back;             // (within a rounding of the sums)
            while (back < 0 && w[at] == 0.0) ++at;
            const uint64_t x = list[back >= 0 ? back : at];
            put_draw(a, row, d, token_of(x), ((double)logit_of(x) - (double)top) / (double)set.T - log_total);
        }
    }
}

// Draws of a list of n entries in the tokens' order that has the k largest, or all that can be kept (one CTA alone).  whole: the mass that
// top-p is of; 0: the k largest entries'.  room: 2 MOST numbers; sums, scan: one for each warp; count: kBins; scale: of bins below top that
// hold the list's logits.
template <int NT, int MOST>
__device__ void draw_listed(const uint64_t *list, uint64_t *room, double *sums, uint32_t *count, uint32_t *scan, const SampleArgs &a, int row,
                            const Settings &set, int n, double whole, const Mass &mass, float top, float scale) {
    __shared__ uint32_t first_out;
    uint64_t *down = room, *tmp = room + MOST;
    // ---- in falling order: what is kept is a prefix, so everything from an entry on
    for (int i = threadIdx.x; i < n; i += NT) down[i] = list[i];
    order_down<NT, kBins>(down, tmp, n, count, scan, [&](uint64_t e) { return bin_below(top, logit_of(e), scale); });
    const int most = set.k ? min(n, set.k) : n;
    if (threadIdx.x == 0) first_out = (uint32_t)most;
    double *w = reinterpret_cast<double *>(tmp);
#pragma unroll 4
    for (int i = threadIdx.x; i < most; i += NT) w[i] = mass.of(logit_of(down[i]));
    __syncthreads();
    // a thread's entries lie side by side, an odd number of them (an even one would send a warp's lanes to few banks)
    int each = (most + NT - 1) / NT | 1, begin = min((int)threadIdx.x * each, most), end = min(begin + each, most);
    double total, mine = 0.0;
    for (int i = begin; i < end; ++i) mine += w[i];
    double upto = before<NT>(mine, &total, sums);  // (barriers)
    if (whole != 0.0) total = whole;
    const double goal = set.p < 1.f ? (double)set.p * total : (double)CUDART_INF_F;
    for (int i = begin; i < end; ++i) {
        if (!(upto < goal) || !(w[i] >= (double)set.m) || w[i] == 0.0) {
            atomicMin(&first_out, (uint32_t)i);
            break;
        }
        upto += w[i];
    }
    __syncthreads();
    const uint64_t least = down[first_out - 1];
    // ---- in the tokens' order: cumulative masses of what is kept
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += NT) w[i] = list[i] >= least ? mass.of(logit_of(list[i])) : 0.0;
    draw_kept<NT, MOST>(list, w, reinterpret_cast<double *>(room), sums, a, row, set, n, top);
}

// The same for a prefix of top-p or min-p whose end lies in the bins from `inside` on, of width 1 / scale below top: only these bins'
// entries are compared with one another.  False if they are more than `most`, up to NT (nothing is drawn then).  near: 2 most numbers.
template <int NT, int MOST>
__device__ bool draw_prefix(const uint64_t *list, uint64_t *room, double *sums, uint64_t *near, int most, const SampleArgs &a, int row,
                            const Settings &set, int n, double whole, const Mass &mass, float top, float scale, int inside) {
    double *near_mass = reinterpret_cast<double *>(near + most);
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    double *w = reinterpret_cast<double *>(room), *upto_of = w + MOST;
    const double m = (double)set.m;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += NT) {
        const double x = mass.of(logit_of(list[i]));
        w[i] = x >= m ? x : 0.0;                   // (what is below m has no part in a larger entry's sum)
    }
    if (set.p < 1.f) {
        const float sure = Range(top, scale, inside, kBins - 1).above;
        const int each = (n + NT - 1) / NT | 1, begin = min((int)threadIdx.x * each, n), end = min(begin + each, n);
        double above = 0.0;
        uint32_t mine = 0, total;
        __syncthreads();
        for (int i = begin; i < end; ++i) {
            const bool in = logit_of(list[i]) >= sure;
            if (in) above += w[i];
            mine += !in;
        }
        uint32_t at = before<NT>(mine, &total, reinterpret_cast<uint32_t *>(sums));
        if (total > (uint32_t)most) return false;
        above = over_cta<NT>(above, add, sums);    // (barriers)
        for (int i = begin; mine && i < end; ++i)
            if (logit_of(list[i]) < sure) {
                near[at] = list[i];
                near_mass[at++] = w[i];
            }
        __syncthreads();
        // an entry stays while what is larger has less than the goal; the least one that does, or none of these
        const double goal = (double)set.p * whole;
        uint64_t e = ~0ull;
        if (threadIdx.x < total) {
            const uint64_t own = near[threadIdx.x];
            double upto = above;
#pragma unroll 4
            for (int i = 0; i < (int)total; ++i) upto += near[i] > own ? near_mass[i] : 0.0;
            if (upto < goal) e = own;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) e = min(e, (uint64_t)__shfl_xor_sync(kFull, (unsigned long long)e, o));
        uint64_t *least_of = reinterpret_cast<uint64_t *>(sums);
        if (lane == 0) least_of[warp] = e;
        __syncthreads();
        uint64_t least = ~0ull;
#pragma unroll
        for (int v = 0; v < NT / 32; ++v) least = min(least, least_of[v]);
        for (int i = begin; i < end; ++i)
            if (list[i] < least && logit_of(list[i]) < sure) w[i] = 0.0;
    }
    draw_kept<NT, MOST>(list, w, upto_of, sums, a, row, set, n, top);
    return true;
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
        for (int e = 0; e < kPer<T>; ++e) m[e] = mass.of(x[e]);
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) {
            if (!(m[e] >= least) || !(x[e] > z_cut || (x[e] == z_cut && t + e <= cut.token))) m[e] = 0.0;
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
__device__ void draw_cut(const SampleArgs &a, float4 *mem, Shared &sh) {
    const int row = blockIdx.x / a.ctas, rank = blockIdx.x - row * a.ctas;
    Settings set;
    if (settings_of(a, row, set) != kCut) return;
    begun_arrive(a.ctas);
    const T *at = static_cast<const T *>(a.logits) + (int64_t)row * a.stride;
    Row<T> r = {share<T>(at, a.V, rank, a.per), mem, sh, reinterpret_cast<uint64_t *>(mem + a.words), a.list_room, a.ctas, rank, 0, 0, 0.f, 0.f};
    Mass::fill(sh.table);
    if (!bring<T>(r, at, mem, a.status)) {
        if (rank == 0)
            for (int d = threadIdx.x; d < a.draws; d += kThreads) no_draw(a, row, d, 0);
        return;
    }
    const Mass mass(set.T, r.top, sh.table);
    double whole_mass = 0.0;
    int n = -1;
    float finer = 0.f;                             // scale of bins that hold the list's logits alone
    float scale = 0.f;
    int inside = 0, last = kBins - 1;
    if (set.k == 0) {
        n = list_mass(r, set.p, set.m, set.T, mass, &whole_mass, &scale, &inside, &last);
        finer = scale * ((float)kBins / (float)(last + 1));
    } else if (set.k <= kTop<T>) {
        n = list_top(r, set.k, &finer);
    }
    if (n >= 0) {
        if (rank == 0 && (set.k || !draw_prefix<kThreads, kList>(r.list, r.tmp(), sh.sums, reinterpret_cast<uint64_t *>(sh.hist), kNear, a, row, set, n,
                                                                 whole_mass, mass, r.top, scale, inside)))
            draw_listed<kThreads, kList>(r.list, r.tmp(), sh.sums, sh.hist[0].count, reinterpret_cast<uint32_t *>(sh.scan), a, row, set, n,
                                         whole_mass, mass, r.top, finer);
        return;
    }
    Cut cut = {kKeyMasked, -1};                    // everything above -inf
    // a prefix longer than the list: only where it ends is put in order (64 rows of 128256 fp32 with settings of their own: 86 us by
    // levels of bins, 67 so; where the list holds the prefix, it in order is faster: 512 rows of such, top-p 0.95, 447 us against 720)
    if (set.k == 0 && set.p < 1.f && inside > 0 && last < kBins - 1 &&
        cut_in_bins(r, scale, inside, last, (double)set.p * whole_mass, mass, &cut)) {
        draw_shared(r, a, row, set, cut, mass);
        return;
    }
    const Whole whole = {mass, (double)(1ull << (30 + __clz(a.V - 1 | 1)))};
    if (set.k) cut = cut_at<false>(r, cut, (uint32_t)set.k, 0.f, whole, 2.f * (r.top - r.low));
    if (set.p < 1.f) cut = cut_at<true>(r, cut, 0, set.p, whole, 64.f * 0.6931472f * set.T);
    draw_shared(r, a, row, set, cut, mass);
}

// 512 rows of 128256 fp32 with top-p 0.95 at temperature 0.9 take 392 us (their bytes 40; at temperature 1 prefixes are longer, 561) and 113 warp
// instructions an element, 17 to bring it, 51 for its mass in 64 bits and its bin, 38 to list; part of each are the exchanges' some hundreds a
// thread.  No pipe is full (issue slots 56 %, ALU 40 %): phases stand behind one another, with barriers of the cluster between them, and two CTAs
// of an SM cover each other in part.  A few rows are a chain: one of these 22 us, of which 3 bring it, 6.5 are masses
// and bins, 5.5 the list, 6.5 its end and the draw.  Shares of 64 KB, so that two CTAs fit an SM (64 rows in clusters of 4 and of 8: 63 and 64 us; 512 rows 417 and 392).
//
// Beside k_draw, whose rows are others: its CTAs have all waited for what came before them when this kernel is launched, so this one
// need not; but it ends after k_draw has, as what comes next waits for this kernel alone.
template <class T>
__global__ void __launch_bounds__(kThreads, 2) k_draw_cut(SampleArgs a) {
    extern __shared__ float4 mem[];
    __shared__ Shared sh;
    if (!a.beside) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    }
    draw_cut<T>(a, mem, sh);
    if (a.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ------------------------------------------------------------------------------------ rows of one pass
constexpr int kOnce = 256;                         // threads
constexpr int kOnceResident = 3;                   // CTAs of an SM
constexpr int kOnceTop = 512;                      // top-k, at most
constexpr int kShareTop = 128;                     // the same where rows have their own, and CTAs of a row are not chosen by it
constexpr int kBatches = DSBD_MAX_ROW_BYTES / 2 / 1024 + 16;           // of 1024 tokens, of the longest row (bf16)
using DrawList = TopList<kOnce, 4, 2048, 1536>;

struct Report {
    double mass;
    float top;
    uint32_t listed;                               // ~0: a NaN or +inf
};

struct Batches {
    double upto[kBatches];
    float top[kBatches];
};

struct DrawShared {
    double table[64];
    Told<Report> told;
    union {
        DrawList list;
        Batches batch;
    };
    double sums[kOnce / 32];
};

// Draws of a row without cuts: each CTA those of its share.
template <class T>
__device__ void draw_plain(DrawShared &sh, const SampleArgs &a, int row, int rank, const T *at, const Settings &set) {
    constexpr int P = kPer<T>, D = kDeep<T>, kBatch = D * kOnce;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    const Share s = share<T>(at, a.V, rank, a.per);
    Batches &batch = sh.batch;
    Mass mass(set.T, 0.f, sh.table);
    // a warp's batch: its mass and largest logit.  Batches are in the tokens' order: number w0 / kBatch * warps + warp.
    bool good = true;
    int batches = 0;
    for (int w0 = 0; w0 < s.words; w0 += kBatch, batches += kOnce / 32) {
        float4 raw[D];
        load_batch<T, kOnce>(raw, at, s, w0);
        float top = -CUDART_INF_F;
#pragma unroll
        for (int u = 0; u < D; ++u) {
            float x[P];
            unpack(raw[u], x);
#pragma unroll
            for (int e = 0; e < P; ++e) top = max_nan(top, x[e]);
        }
        good &= top < CUDART_INF_F;
        top = warp_most(top < CUDART_INF_F ? top : -CUDART_INF_F);
        double sum = 0.0;
        if (top > -CUDART_INF_F) {
            mass.relative_to(top);
#pragma unroll
            for (int u = 0; u < D; ++u) {
                float x[P];
                unpack(raw[u], x);
                sum += mass.of_word(x);
            }
            sum = warp_sum(sum);
        }
        if (lane == 0) {
            batch.upto[batches + warp] = sum;
            batch.top[batches + warp] = top;
        }
    }
    good = __syncthreads_and(good);
    // the share's largest logit, the batches' masses relative to it, and their cumulative sums
    float top = -CUDART_INF_F;
    for (int b = lane; b < batches; b += 32) top = fmaxf(top, batch.top[b]);
    top = warp_most(top);
    Mass rel = mass;
    rel.relative_to(top);
    __syncthreads();
    for (int b = threadIdx.x; b < batches; b += kOnce) {
        const double m = batch.upto[b] * rel.of(batch.top[b]);
        batch.upto[b] = m;
        if (m == 0.0) batch.top[b] = -CUDART_INF_F;
    }
    __syncthreads();
    if (warp == 0) {
        const int each = (batches + 31) / 32, b0 = min(lane * each, batches), b1 = min(b0 + each, batches);
        double sum = 0.0;
        for (int b = b0; b < b1; ++b) sum += batch.upto[b];
        double up = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double x = __shfl_up_sync(kFull, up, o);
            if (lane >= o) up += x;
        }
        sum = __shfl_up_sync(kFull, up, 1);
        if (lane == 0) sum = 0.0;
        for (int b = b0; b < b1; ++b) {
            sum += batch.upto[b];
            batch.upto[b] = sum;
        }
    }
    __syncthreads();
    begun_wait(a.ctas);
    int turn = 0;
    const double mine = batches ? batch.upto[batches - 1] : 0.0;
    const Report own = {mine, top, good ? 0u : ~0u};
    const Report *all = tell(own, sh.told, turn, a.ctas, rank);
    float most = all[0].top;
    for (int c = 0; c < a.ctas; ++c) {
        good &= all[c].listed == 0;
        most = fmaxf(most, all[c].top);
    }
    if (!good || most == -CUDART_INF_F) {
        if (rank == 0) {
            for (int d = threadIdx.x; d < a.draws; d += kOnce) no_draw(a, row, d, 0);
            if (threadIdx.x == 0) report(a.status, good ? DSBD_DEV_EXHAUSTED : DSBD_DEV_BAD_LOGIT);
        }
        return;
    }
    // where the shares begin and end, by the same roundings in every CTA
    Mass between = mass;
    between.relative_to(most);
    double begin = 0.0, total = 0.0;
    for (int c = 0; c < a.ctas; ++c) {
        if (c == rank) begin = total;
        total = __dadd_rn(total, __dmul_rn(all[c].mass, between.of(all[c].top)));
    }
    const double unit = between.of(top), end = __dadd_rn(begin, __dmul_rn(mine, unit));
    const double log_total = log(total);
    for (int d = warp; d < a.draws; d += kOnce / 32) {
        const float u = a.uniform[(int64_t)row * a.draws + d];
        if (!(u >= 0.f && u <= 1.f)) {
            if (rank == 0 && lane == 0) no_draw(a, row, d, DSBD_DEV_BAD_PARAM);
            continue;
        }
        const double t = target(u, total);
        if (!(begin <= t && t < end)) continue;
        // the first batch that ends beyond t
        int b = 0;
        for (int i = lane; i < batches; i += 32) b += __dadd_rn(begin, __dmul_rn(batch.upto[i], unit)) <= t;
        b = min((int)__reduce_add_sync(kFull, (unsigned)b), batches - 1);
        if (batch.top[b] == -CUDART_INF_F) {
            // (t lies within a rounding of the sums before a batch without mass: the last one with some)
            int before_ = -1, behind = batches;
            for (int i = lane; i < batches; i += 32)
                if (batch.top[i] > -CUDART_INF_F) {
                    if (i < b) before_ = max(before_, i);
                    else behind = min(behind, i);
                }
            before_ = __reduce_max_sync(kFull, before_);
            behind = __reduce_min_sync(kFull, behind);
            b = before_ >= 0 ? before_ : behind;
        }
        const float from = batch.top[b];
        mass.relative_to(from);
        // what is left of t in the batch, relative to its largest logit
        const double left = ((t - begin) / unit - (b ? batch.upto[b - 1] : 0.0)) / rel.of(from);
        double done = 0.0;
        int token = -1;
        float z = 0.f;
        const int first = b / (kOnce / 32) * kBatch + b % (kOnce / 32) * D * 32;
        for (int v = 0; v < D; ++v) {
            const int w = first + v * 32 + lane;
            float x[P];
            unpack(w < s.words ? load_word(at, s, w) : masked_word<T>(), x);
            double m[P], here = 0.0;
#pragma unroll
            for (int e = 0; e < P; ++e) {
                m[e] = mass.of(x[e]);
                here += m[e];
            }
            double up = here;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double y = __shfl_up_sync(kFull, up, o);
                if (lane >= o) up += y;
            }
            // the first lane that goes beyond; where rounding lets none, the last one with a mass
            const unsigned beyond = __ballot_sync(kFull, done + up > left && here > 0.0), some = __ballot_sync(kFull, here > 0.0);
            if (some) {
                const int who = beyond ? __ffs(beyond) - 1 : 31 - __clz(some);
                if (lane == who) {
                    double c = done + (up - here);
#pragma unroll
                    for (int e = 0; e < P; ++e)
                        if (m[e] != 0.0 && !(c > left)) {
                            token = s.first + w * P - s.mis + e;
                            z = x[e];
                            c += m[e];
                        }
                }
                token = __shfl_sync(kFull, token, who);
                z = __shfl_sync(kFull, z, who);
            }
            if (beyond) break;
            done += __shfl_sync(kFull, up, 31);
        }
        if (lane == 0) put_draw(a, row, d, token, ((double)z - (double)most) / (double)set.T - log_total);
    }
}

// Draws of a list that has the k largest (in no order), one CTA alone.
__device__ void draw_few(DrawShared &sh, const SampleArgs &a, int row, const Settings &set) {
    DrawList &list = sh.list;
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, n = (int)list.listed;
    list.sort();
    const float top = logit_of(list.list[0]);
    const Mass mass(set.T, top, sh.table);
    if (set.k > 32) {
        // in the tokens' order, as draw_listed wants them
        uint64_t *by_token = reinterpret_cast<uint64_t *>(list.hot), *tmp = by_token + kOnceTop;
        const int kept = min(n, set.k);
        for (int i = threadIdx.x; i < kept; i += kOnce) by_token[i] = (list.list[i] << 32) | (list.list[i] >> 32);
        const float per_bin = (float)kBins / (float)a.V, low = logit_of(list.list[kept - 1]);
        order_down<kOnce, kBins>(by_token, tmp, kept, list.count, list.scan,
                                 [&](uint64_t x) { return min((int)((float)~(uint32_t)(x >> 32) * per_bin), kBins - 1); });
        for (int i = threadIdx.x; i < kept; i += kOnce) list.list[i] = (by_token[i] << 32) | (by_token[i] >> 32);
        draw_listed<kOnce, kOnceTop>(list.list, by_token, sh.sums, list.count, list.scan, a, row, set, kept, 0.0, mass, top, bins_over(top - low));
        return;
    }
    // an entry to a lane; the warps share the draws
    const int kept = min(n, set.k);
    const uint64_t mine = lane < kept ? list.list[lane] : 0;
    double w = lane < kept ? mass.of(logit_of(mine)) : 0.0, upto = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double x = __shfl_up_sync(kFull, upto, o);
        if (lane >= o) upto += x;
    }
    double below = __shfl_up_sync(kFull, upto, 1), total = __shfl_sync(kFull, upto, 31);
    if (lane == 0) below = 0.0;
    const bool out = lane >= kept || (set.p < 1.f && !(below < (double)set.p * total)) || !(w >= (double)set.m) || w == 0.0;
    const unsigned cut = __ballot_sync(kFull, out);
    const int in = cut ? __ffs(cut) - 1 : 32;
    if (lane >= in) w = 0.0;
    const uint32_t token = lane < in ? (uint32_t)token_of(mine) : 0x7fffffffu;
    // cumulative masses in the tokens' order
    upto = 0.0;
    total = 0.0;
    for (int j = 0; j < in; ++j) {
        const double x = __shfl_sync(kFull, w, j);
        upto += __shfl_sync(kFull, token, j) <= token ? x : 0.0;
        total += x;
    }
    // (by another order of additions the last sum may differ from the whole in its last bit)
    const uint32_t last = __reduce_max_sync(kFull, lane < in ? token : 0u);
    const double log_total = log(total);
    for (int d = warp; d < a.draws; d += kOnce / 32) {
        const float u = a.uniform[(int64_t)row * a.draws + d];
        if (!(u >= 0.f && u <= 1.f)) {
            if (lane == 0) no_draw(a, row, d, DSBD_DEV_BAD_PARAM);
            continue;
        }
        const double t = target(u, total);
        const uint32_t found = __reduce_min_sync(kFull, lane < in && (upto > t || token == last) ? token : 0x7fffffffu);
        if (lane < in && token == found) put_draw(a, row, d, (int)token, ((double)logit_of(mine) - (double)top) / (double)set.T - log_total);
    }
}

// Rows without cuts take the time of the 64-bit exponentials of all tokens (30 warp instructions an element, of which 12 on the FP64 pipe: 512 rows of
// 128256, 8 draws each, fp32 110 us of 40 at the copy rate, bf16 102 of 20); exponentials in 32 bits would stream, but are off by more than an
// improbable token's cell.  No pipe is full (issue 56 %, FP64 40 %): it is the latency of dependent steps, and of loads of which none are in flight
// while a batch is worked on, with three CTAs of an SM.  Rows with a short top-k and those at temperature 0 take what k_top takes, a chain of words,
// bounds, exchange and order: one row of 32000 with top-k 10 and top-p 0.8 10 us; 64 rows of 128256 with top-k 50 fp32 25, bf16 23, at temperature 0
// 17 and 15; 512 rows with top-k 20 fp32 78 (of 40), bf16 71, with top-k 100 98 and 90, at temperature 0 fp32 69.
template <class T>
__global__ void __launch_bounds__(kOnce, kOnceResident) k_draw(SampleArgs a) {
    extern __shared__ float4 mem[];
    DrawShared &sh = *reinterpret_cast<DrawShared *>(mem);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int row = blockIdx.x / a.ctas, rank = blockIdx.x - row * a.ctas;
    Settings set;
    const Kind kind = settings_of(a, row, set);
    if (kind == kCut) return;
    if (kind == kBad) {
        if (rank == 0)
            for (int d = threadIdx.x; d < a.draws; d += kOnce) no_draw(a, row, d, DSBD_DEV_BAD_PARAM);
        return;
    }
    begun_arrive(a.ctas);
    Mass::fill(sh.table);
    __syncthreads();
    const T *at = static_cast<const T *>(a.logits) + (int64_t)row * a.stride;
    if (kind == kPlain) {
        draw_plain(sh, a, row, rank, at, set);
        return;
    }
    const uint32_t K = kind == kGreedy ? 1 : (uint32_t)set.k;
    Rest rest;
    Sum cleared = {-CUDART_INF_F, 0.0};
    const bool good = collect<T, false>(sh.list, at, share<T>(at, a.V, rank, a.per), K, a.ctas > 1, 0.f, rest, cleared);
    begun_wait(a.ctas);
    int turn = 0;
    const Report own = {0.0, 0.f, good ? sh.list.listed : ~0u};
    const Report *all = tell(own, sh.told, turn, a.ctas, rank);
    bool bad = false;
    uint64_t n = 0;
    for (int c = 0; c < a.ctas; ++c) {
        bad |= all[c].listed == ~0u;
        n += all[c].listed;
    }
    const bool over = n > DrawList::kList;
    if (rank == 0 && !bad && !over) {
        uint32_t to = all[0].listed;
        for (int c = 1; c < a.ctas; ++c) {
            const uint64_t *from = cg::this_cluster().map_shared_rank(&sh.list.list[0], c);
            for (uint32_t i = threadIdx.x; i < all[c].listed; i += kOnce) sh.list.list[to + i] = from[i];
            to += all[c].listed;
        }
        if (threadIdx.x == 0) sh.list.listed = to;
    }
    cluster_barrier(a.ctas);                       // (rank 0 has the lists)
    if (rank) return;
    if (bad || n == 0) {
        for (int d = threadIdx.x; d < a.draws; d += kOnce) no_draw(a, row, d, 0);
        if (threadIdx.x == 0) report(a.status, bad ? DSBD_DEV_BAD_LOGIT : DSBD_DEV_EXHAUSTED);
        return;
    }
    if (over) {
        select_row<T, false>(sh.list, at, a.V, K, 0.f, rest);
    } else {
        sh.list.clear<false>(sh.list.entries_bound(K), 0.f, cleared);
    }
    if (kind == kGreedy) {
        if (threadIdx.x < 32) {
            uint64_t best = 0;
            for (int i = threadIdx.x; i < (int)sh.list.listed; i += 32) best = sh.list.list[i] > best ? sh.list.list[i] : best;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const uint64_t x = __shfl_xor_sync(kFull, best, o);
                best = x > best ? x : best;
            }
            for (int d = threadIdx.x; d < a.draws; d += 32) {
                const float u = a.uniform[(int64_t)row * a.draws + d];
                if (u >= 0.f && u <= 1.f) put_draw(a, row, d, token_of(best), 0.0);
                else no_draw(a, row, d, DSBD_DEV_BAD_PARAM);
            }
        }
        return;
    }
    draw_few(sh, a, row, set);
}

// k_draw_cut: the longest share with a whole list beside it, in 16-byte words; the most shared memory of a CTA.
constexpr int kWholeList = 160 * 1024 / 16;
constexpr int kCutBytes = std::max(kWholeList * 16 + kList * 8, kLongestShare * 16 + kList / 2 * 8);
static_assert(kWholeList >= kList && kCutBytes + sizeof(Shared) <= 227 * 1024, "");

// CTAs of a row in k_draw: lists of up to K entries and a half more from each.
inline Plan plan_once(const dsbd_rows_t *r, int K) {
    int most = kMaxCtas;
    while (most > 1 && 3 * (int64_t)K * most > 2 * DrawList::kList) most /= 2;
    return plan_waves(r, 148 * kOnceResident, 24000, kOnce * 16, most);
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
    SampleArgs a = {};
    a.logits = rows->logits; a.stride = rows->row_stride; a.V = rows->V; a.draws = p->draws;
    a.temperature = p->temperature; a.top_p = p->top_p; a.min_p = p->min_p; a.top_k = p->top_k;
    a.temperature_r = p->temperature_r; a.top_p_r = p->top_p_r; a.min_p_r = p->min_p_r; a.top_k_r = p->top_k_r;
    a.uniform = uniform; a.token = token; a.logp = logp; a.status = status;
    a.list_most = p->top_k_r ? kShareTop : kOnceTop;
    // the kernels that rows of these settings may need; each leaves the other's rows alone
    const bool k_off = !p->top_k_r && (p->top_k <= 0 || p->top_k >= rows->V), no_cut = p->top_p >= 1.f && p->min_p == 0.f;
    bool once = true, cut = true;
    if (!p->temperature_r && p->temperature == 0.f) cut = false;
    else if (!p->top_k_r && !k_off) (p->top_k <= kOnceTop ? cut : once) = false;
    else if (k_off && !p->top_p_r && !p->min_p_r) (no_cut ? cut : once) = false;
    if (!cut || p->temperature_r || p->top_p_r || p->min_p_r) once = true;      // (settings out of range are k_draw's)
    if (once) {
        const Plan plan = plan_once(rows, p->top_k_r ? kShareTop : k_off ? 1 : p->top_k < kOnceTop ? p->top_k : kOnceTop);
        a.ctas = plan.ctas;
        a.per = plan.per;
        rc = rows->dtype == DSBD_DTYPE_F32 ? launch<sizeof(DrawShared), kOnce>(k_draw<float>, rows->rows, plan, sizeof(DrawShared), a, stream)
                                           : launch<sizeof(DrawShared), kOnce>(k_draw<__nv_bfloat16>, rows->rows, plan, sizeof(DrawShared), a, stream);
        if (rc) return rc;
    }
    if (!cut) return DSBD_OK;
    const Plan plan = plan_for(rows);
    a.beside = once;
    a.ctas = plan.ctas;
    a.per = plan.per;
    // the share, where the list is put in order and its masses are later, and the list; half as long beside the longest shares
    a.list_room = plan.words <= kWholeList ? kList : kList / 2;
    a.words = plan.words > kList ? plan.words : kList;
    const size_t bytes = (size_t)a.words * 16 + (size_t)a.list_room * 8;
    return rows->dtype == DSBD_DTYPE_F32 ? launch<kCutBytes>(k_draw_cut<float>, rows->rows, plan, bytes, a, stream)
                                         : launch<kCutBytes>(k_draw_cut<__nv_bfloat16>, rows->rows, plan, bytes, a, stream);
}
