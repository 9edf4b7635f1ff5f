// Between a model's QKV projection and its cache and attention: the rotation of queries and keys by position with the
// norms of the heads, the append of a chunk's keys and values to the paged cache, the positions of a forest's nodes, and
// the table of cosines and sines that the rotations read.
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>

#include "dsbd_common.cuh"

using namespace dsbd;

namespace {

constexpr int kMaxRot = 128;
constexpr int kThreads = 128;

// Launched while the kernel before it may still run: wait for that one's results, then let the next one come (which waits
// for these in turn).
__device__ __forceinline__ void pdl_wait() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// ------------------------------------------------------------------------------------------ table
struct Frequencies { double f[kMaxRot / 2]; };

__global__ void __launch_bounds__(kThreads)
k_rope_table(Frequencies fr, double attention, int half, int64_t n, float *__restrict__ table) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= n) return;
    const int64_t pos = i / half;
    const int j = (int)(i - pos * half);
    double s, c;
    sincos((double)pos * fr.f[j], &s, &c);
    table[pos * 2 * half + j] = (float)(c * attention);
    table[pos * 2 * half + half + j] = (float)(s * attention);
}

int frequencies(const dsbd_rope_scaling_t *s, int rot, double *f, double *attention) {
    if (!s || !f || rot < 2 || rot > kMaxRot || rot % 2 || !(s->base > 1.0) || !std::isfinite(s->base)) return DSBD_ERR_INVALID_ARG;
    const int kind = s->kind;
    if (kind < DSBD_ROPE_PLAIN || kind > DSBD_ROPE_RAMP) return DSBD_ERR_UNSUPPORTED;
    if (kind != DSBD_ROPE_PLAIN && !(s->factor >= 1.0 && std::isfinite(s->factor))) return DSBD_ERR_INVALID_ARG;
    if (kind == DSBD_ROPE_BASE && rot == 2) return DSBD_ERR_INVALID_ARG;
    if ((kind == DSBD_ROPE_WAVELENGTH || kind == DSBD_ROPE_RAMP) &&
        !(s->original > 0.0 && s->low > 0.0 && s->high > s->low && std::isfinite(s->original) && std::isfinite(s->high)))
        return DSBD_ERR_INVALID_ARG;
    if (kind == DSBD_ROPE_RAMP && !(s->attention >= 0.0 && std::isfinite(s->attention))) return DSBD_ERR_INVALID_ARG;
    const double kPi = 3.14159265358979323846;
    const double base = kind == DSBD_ROPE_BASE ? s->base * pow(s->factor, (double)rot / (rot - 2)) : s->base;
    // RAMP: dimension at which `turns` turns fit into the trained context
    auto dimension = [&](double turns) { return rot * log(s->original / (turns * 2.0 * kPi)) / (2.0 * log(s->base)); };
    double lo = 0.0, hi = 0.0;
    if (kind == DSBD_ROPE_RAMP) {
        lo = std::max(floor(dimension(s->high)), 0.0);
        hi = std::min(ceil(dimension(s->low)), (double)rot - 1.0);
        if (hi <= lo) hi = lo + 0.001;
    }
    for (int i = 0; i < rot / 2; ++i) {
        double w = pow(base, -2.0 * i / rot);
        if (kind == DSBD_ROPE_LINEAR) w /= s->factor;
        if (kind == DSBD_ROPE_WAVELENGTH) {
            const double turns = s->original * w / (2.0 * kPi);
            const double keep = std::min(std::max((turns - s->low) / (s->high - s->low), 0.0), 1.0);
            w = keep * w + (1.0 - keep) * w / s->factor;
        }
        if (kind == DSBD_ROPE_RAMP) {
            const double scaled = std::min(std::max((i - lo) / (hi - lo), 0.0), 1.0);
            w = scaled * w / s->factor + (1.0 - scaled) * w;
        }
        f[i] = w;
    }
    if (attention) *attention = kind != DSBD_ROPE_RAMP ? 1.0 : s->attention > 0.0 ? s->attention : 0.1 * log(s->factor) + 1.0;
    return DSBD_OK;
}

// ------------------------------------------------------------------------------------------ positions
constexpr int kTreeWarps = 4, kTreeSmem = 1056;     // dsbd_forest_build makes trees of at most 1025 nodes

// A warp to a tree: its parents go to shared memory, every lane walks up from its nodes (a dependent chain of
// shared-memory look-ups instead of one of global loads).  Parents come before their children, so a walk ends.  Walks of large
// trees would cost their nodes times their depth; those are done 32 nodes at a time behind what is done already.
// (No __restrict__: the blocks may be resident while the kernel before, dsbd_forest_build's for one, writes the forest, and
// data that is written meanwhile must not be read by non-coherent loads.)
__global__ void __launch_bounds__(kTreeWarps * 32)
k_forest_positions(int B, int N, const int32_t *node_off, const int32_t *parent, const int64_t *prefix_off, int32_t *position,
                   int32_t *status) {
    __shared__ int par_s[kTreeWarps][kTreeSmem];
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, b = blockIdx.x * kTreeWarps + warp;
    if (b >= B) return;
    const int lo = node_off[b], hi = node_off[b + 1];
    const int64_t L = prefix_off[b + 1] - prefix_off[b];
    if (lo < 0 || hi > N || lo > hi || L < 0 || L > (int64_t)INT32_MAX - N) {
        if (lane == 0) report(status, DSBD_DEV_BAD_FOREST);
        return;
    }
    const int n = hi - lo;
    int *par = par_s[warp];
    if (n <= kTreeSmem) {
        for (int i = lane; i < n; i += 32) par[i] = parent[lo + i] - lo;
        __syncwarp();
        for (int i = lane; i < n; i += 32) {
            int depth = 0;
            for (int j = i; ;) {
                const int p = par[j];
                if (p < 0 || p >= j) {
                    if (j == i && (i != 0 || p != -1 - lo)) report(status, DSBD_DEV_BAD_FOREST);
                    break;
                }
                ++depth;
                j = p;
            }
            position[lo + i] = (int)L + depth;
        }
        return;
    }
    // 32 nodes at a time, whose ancestors among the 32 are found by doubling; an ancestor before them has its position already
    for (int base = 0; base < n; base += 32) {
        const int i = base + lane;
        int up = -1, depth = 0;                      // an ancestor of node i, and how far above it
        if (i < n) {
            const int p = parent[lo + i] - lo;
            if (p >= 0 && p < i) { up = p; depth = 1; }
            else if (i != 0 || p != -1 - lo) report(status, DSBD_DEV_BAD_FOREST);
        }
#pragma unroll
        for (int r = 0; r < 5; ++r) {
            const int src = up >= base ? up - base : lane;
            const int next = __shfl_sync(kFull, up, src), more = __shfl_sync(kFull, depth, src);
            if (up >= base) { up = next; depth += more; }
        }
        if (i < n) position[lo + i] = (up >= 0 ? position[lo + up] : (int)L) + depth;
        __syncwarp();
    }
}

// ------------------------------------------------------------------------------------------ rotation and append
// Four neighbouring values of a row, as they lie in memory and widened to fp32.
template <class T> struct Four;
template <> struct Four<float> {
    using Raw = uint4;
    __device__ static void widen(const Raw &v, float *x) {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
    __device__ static Raw narrow(const float *x) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};
template <> struct Four<__nv_bfloat16> {
    using Raw = uint2;
    __device__ static void widen(const Raw &v, float *x) {
        x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
        x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
    }
    __device__ static Raw narrow(const float *x) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
        return make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
    }
};

// Two fp32 operations an instruction (sm_100): the kernel below has 65 % of its issue slots full with single ones.
struct F2 { float x, y; };
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    F2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "mul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
// (u, v) turned, two pairs: (u c - v s, v c + u s); ms = -s
__device__ __forceinline__ void turn2(F2 &u, F2 &v, F2 c, F2 s, F2 ms) {
    const F2 t = fma2(v, ms, mul2(u, c));
    v = fma2(u, s, mul2(v, c));
    u = t;
}

struct RopeArgs {
    int T, Hq, Hkv;
    int q_pieces, k_pieces, pieces;                  // pieces of a few warp steps: of q, of k; all of a token (v's too)
    int per_warp, parts;                             // pieces a warp takes, warps of a token
    int rot, layout, n_positions;
    float eps;
    const float *table, *q_norm, *k_norm;
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
    void *q_out, *k_out;                             // k_out: not with the append
    const int32_t *position;                         // rotation alone
    // append
    int B;
    int64_t max_len, n_pages;
    const int32_t *new_off, *page_table;
    const int64_t *prefix_off, *page_off;
    void *k_pool, *v_pool;
    int32_t *status;
};

// Steps of a piece, whose loads (64 bytes a lane) are in flight together: four of bf16, two of fp32 (at 64 registers).
__host__ __device__ constexpr int unroll(int size) { return size == 2 ? 4 : 2; }

// The sequence of row t: the largest b with new_off[b] <= t, by a warp, 32 probes at a time.
__device__ __forceinline__ int find_sequence(const int32_t *new_off, int B, int t, int lane) {
    int lo = 0, n = B;                               // the answer is in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32;
        const int at = lo + lane * step;
        const unsigned le = __ballot_sync(kFull, lane * step < n && new_off[at] <= t);
        const int k = le ? 31 - __clz(le) : 0;       // (offsets ascend: the last lane that is not past t)
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

// A warp takes a token and some of its heads, 32 / (d / 8) of them a step, a lane eight values of one: two fours that are each other's
// partners (i and i + rot / 2 in the half layout; neighbours in the interleaved one and behind the rotated part), so that no
// value crosses lanes but the norm's sum.  A token's row of cosines and sines goes to registers once and serves all heads of
// the warp.  Bound by bytes: every value is read and written once.
template <class T, int D, bool APPEND>
__global__ void __launch_bounds__(kThreads, 8)
k_rotate(RopeArgs a) {
    using F = Four<T>;
    using Raw = typename F::Raw;
    constexpr int kLanes = D / 8, kHeads = 32 / kLanes;                 // lanes of a head, heads of a step
    constexpr int kUnroll = unroll(sizeof(T)), kPiece = kHeads * kUnroll;
    pdl_wait();
    const int lane = threadIdx.x & 31, j = lane % kLanes;
    const int64_t job = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const int64_t jobs = (int64_t)a.T * a.parts;
    if (job >= jobs) {
        if (!APPEND) return;
        // what is behind the last token of a page that this call opened: a warp to a sequence, a head and a pool
        const unsigned z = (unsigned)(job - jobs), of_b = z / (2u * a.Hkv), g = (z >> 1) - of_b * a.Hkv;
        if (of_b >= (unsigned)a.B) return;
        const int b = (int)of_b;
        const int n = a.new_off[b + 1] - a.new_off[b];
        const int64_t L = a.prefix_off[b + 1] - a.prefix_off[b], end = L + n;
        const int from = (int)(end % DSBD_PAGE_TOKENS);
        if (n <= 0 || L < 0 || end > a.max_len || from == 0 || end - from < L) return;
        const int64_t p = end / DSBD_PAGE_TOKENS;
        if (p >= a.page_off[b + 1] - a.page_off[b]) return;             // (reported by the tokens' warps)
        const int page = a.page_table[a.page_off[b] + p];
        if (page < 0 || page >= a.n_pages) return;
        T *pool = static_cast<T *>((z & 1) ? a.v_pool : a.k_pool);
        const int left = (DSBD_PAGE_TOKENS - from) * (D * (int)sizeof(T) / 16);      // 16-byte words of a head
        uint4 *dst = reinterpret_cast<uint4 *>(pool + (((int64_t)page * a.Hkv + g) * DSBD_PAGE_TOKENS + from) * D);
        for (int i = lane; i < left; i += 32) dst[i] = make_uint4(0, 0, 0, 0);
        return;
    }
    const int t = a.parts == 1 ? (int)job : (int)((unsigned)job / (unsigned)a.parts);
    int piece = (int)(job - (int64_t)t * a.parts) * a.per_warp;
    const int piece_end = min(piece + a.per_warp, a.pieces);

    // the lane's values: e0 .. e0 + 3 and e1 .. e1 + 3
    const bool by_half = a.layout == DSBD_ROPE_HALF, turned = 8 * j < a.rot;
    const int half = a.rot / 2;
    const int e0 = by_half && turned ? 4 * j : 8 * j, e1 = by_half && turned ? half + 4 * j : 8 * j + 4;

    // where a piece reads: kind 0 q, 1 k, 2 v
    struct Piece { int kind, first, heads; Raw x[kUnroll], y[kUnroll]; };
    auto load = [&](int p) {
        Piece r;
        r.kind = p < a.q_pieces ? 0 : p < a.q_pieces + a.k_pieces ? 1 : 2;
        r.first = (p - (r.kind == 0 ? 0 : r.kind == 1 ? a.q_pieces : a.q_pieces + a.k_pieces)) * kPiece + lane / kLanes;
        r.heads = r.kind == 0 ? a.Hq : a.Hkv;
        const T *src = r.kind == 0 ? static_cast<const T *>(a.q) + t * a.q_stride
                     : r.kind == 1 ? static_cast<const T *>(a.k) + t * a.k_stride : static_cast<const T *>(a.v) + t * a.v_stride;
        src += (int64_t)r.first * D;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            r.x[u] = r.y[u] = Raw{};
            if (r.first + u * kHeads < r.heads) {
                r.x[u] = *reinterpret_cast<const Raw *>(src + u * kHeads * D + e0);
                r.y[u] = *reinterpret_cast<const Raw *>(src + u * kHeads * D + e1);
            }
        }
        return r;
    };
    Piece now = load(piece);

    int64_t pos;
    int64_t row = 0;                                 // of the pools: (page * Hkv) * 64 + slot
    if (APPEND) {
        const int b = find_sequence(a.new_off, a.B, t, lane);
        const int lo = a.new_off[b], hi = a.new_off[b + 1];
        const int64_t L = a.prefix_off[b + 1] - a.prefix_off[b], first_page = a.page_off[b];
        const int64_t n_table = a.page_off[b + 1] - first_page;
        pos = L + (t - lo);
        if (t < lo || t >= hi || L < 0 || pos >= a.max_len || (a.rot && pos >= a.n_positions)) {
            if (lane == 0) report(a.status, DSBD_DEV_BAD_CHUNK);
            return;
        }
        if (pos / DSBD_PAGE_TOKENS >= n_table) {
            if (lane == 0) report(a.status, DSBD_DEV_CAPACITY);
            return;
        }
        const int page = a.page_table[first_page + pos / DSBD_PAGE_TOKENS];
        if (page < 0 || page >= a.n_pages) {
            if (lane == 0) report(a.status, DSBD_DEV_BAD_CHUNK);
            return;
        }
        row = (int64_t)page * a.Hkv * DSBD_PAGE_TOKENS + pos % DSBD_PAGE_TOKENS;
    } else {
        pos = a.position ? a.position[t] : 0;
        if (a.rot && (pos < 0 || pos >= a.n_positions)) {
            if (lane == 0) report(a.status, DSBD_DEV_BAD_CHUNK);
            return;
        }
    }

    // the lane's pairs: 4 j .. 4 j + 3 of the table's row, in either layout
    float4 c = {1.f, 1.f, 1.f, 1.f}, s = {0.f, 0.f, 0.f, 0.f};
    if (turned) {
        const float *cs = a.table + pos * a.rot + 4 * j;
        c = *reinterpret_cast<const float4 *>(cs);
        s = *reinterpret_cast<const float4 *>(cs + half);
    }
    const F2 c0 = {c.x, c.y}, c1 = {c.z, c.w}, s0 = {s.x, s.y}, s1 = {s.z, s.w}, m0 = {-s.x, -s.y}, m1 = {-s.z, -s.w};

    for (;;) {
        const int kind = now.kind;
        const float *norm = kind == 0 ? a.q_norm : kind == 1 ? a.k_norm : nullptr;
        T *dst;
        int64_t pitch = D;
        if (kind == 0) {
            dst = static_cast<T *>(a.q_out) + t * a.q_out_stride;
        } else if (APPEND) {
            dst = static_cast<T *>(kind == 1 ? a.k_pool : a.v_pool) + row * D;
            pitch = DSBD_PAGE_TOKENS * D;
        } else {
            dst = static_cast<T *>(a.k_out) + t * a.k_out_stride;
        }
        dst += now.first * pitch;
        if (kind != 2 && (norm || turned)) {         // (everything else keeps its bits; a head's lanes agree where there is a norm)
            float4 w0 = {1.f, 1.f, 1.f, 1.f}, w1 = {1.f, 1.f, 1.f, 1.f};
            if (norm) {
                w0 = *reinterpret_cast<const float4 *>(norm + e0);
                w1 = *reinterpret_cast<const float4 *>(norm + e1);
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                float x[4], y[4];
                F::widen(now.x[u], x);
                F::widen(now.y[u], y);
                F2 x0 = {x[0], x[1]}, x1 = {x[2], x[3]}, y0 = {y[0], y[1]}, y1 = {y[2], y[3]};
                if (norm) {
                    const F2 q = fma2(x0, x0, fma2(x1, x1, fma2(y0, y0, mul2(y1, y1))));
                    float ss = q.x + q.y;
#pragma unroll
                    for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(kFull, ss, o);
                    const float r = rsqrtf(ss * (1.f / D) + a.eps);
                    const F2 rr = {r, r};
                    x0 = mul2(mul2(x0, rr), F2{w0.x, w0.y}); x1 = mul2(mul2(x1, rr), F2{w0.z, w0.w});
                    y0 = mul2(mul2(y0, rr), F2{w1.x, w1.y}); y1 = mul2(mul2(y1, rr), F2{w1.z, w1.w});
                }
                if (turned) {
                    if (by_half) {
                        turn2(x0, y0, c0, s0, m0);
                        turn2(x1, y1, c1, s1, m1);
                    } else {
                        F2 u0 = {x0.x, x1.x}, v0 = {x0.y, x1.y}, u1 = {y0.x, y1.x}, v1 = {y0.y, y1.y};
                        turn2(u0, v0, c0, s0, m0);
                        turn2(u1, v1, c1, s1, m1);
                        x0 = {u0.x, v0.x}; x1 = {u0.y, v0.y}; y0 = {u1.x, v1.x}; y1 = {u1.y, v1.y};
                    }
                }
                x[0] = x0.x; x[1] = x0.y; x[2] = x1.x; x[3] = x1.y;
                y[0] = y0.x; y[1] = y0.y; y[2] = y1.x; y[3] = y1.y;
                now.x[u] = F::narrow(x);
                now.y[u] = F::narrow(y);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (now.first + u * kHeads < now.heads) {
                *reinterpret_cast<Raw *>(dst + u * kHeads * pitch + e0) = now.x[u];
                *reinterpret_cast<Raw *>(dst + u * kHeads * pitch + e1) = now.y[u];
            }
        if (++piece >= piece_end) break;
        now = load(piece);
    }
}

template <class... Args>
int launch_pdl(void (*kernel)(Args...), int64_t grid, int threads, cudaStream_t stream, Args... args) {
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess ? DSBD_OK : DSBD_ERR_CUDA;
}

int check_desc(const dsbd_attn_desc_t *d) {
    if (!d || d->Hq <= 0 || d->Hkv <= 0 || d->Hq % d->Hkv) return DSBD_ERR_INVALID_ARG;
    if (d->d != 64 && d->d != 128) return DSBD_ERR_UNSUPPORTED;
    if (d->dtype != DSBD_DTYPE_BF16 && d->dtype != DSBD_DTYPE_F32) return DSBD_ERR_UNSUPPORTED;
    return DSBD_OK;
}

int check_rope(const dsbd_rope_t *r, int d) {
    if (!r || r->rot < 0 || r->rot > d || r->rot % 16) return DSBD_ERR_INVALID_ARG;
    if (r->rot && (!r->table || r->n_positions <= 0)) return DSBD_ERR_INVALID_ARG;
    if (r->layout != DSBD_ROPE_HALF && r->layout != DSBD_ROPE_INTERLEAVED) return DSBD_ERR_INVALID_ARG;
    if ((r->q_norm || r->k_norm) && !(r->eps >= 0.f)) return DSBD_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(r->table) | reinterpret_cast<uintptr_t>(r->q_norm) |
         reinterpret_cast<uintptr_t>(r->k_norm)) & 15)
        return DSBD_ERR_UNSUPPORTED;
    return DSBD_OK;
}

// Rows of `heads` heads `stride` elements apart: long enough, and whole 16-byte words.
int check_rows(const void *p, int64_t stride, int heads, const dsbd_attn_desc_t *d) {
    if (!p || stride < (int64_t)heads * d->d) return DSBD_ERR_INVALID_ARG;
    const int size = d->dtype == DSBD_DTYPE_BF16 ? 2 : 4;
    return (reinterpret_cast<uintptr_t>(p) | (uint64_t)(stride * size)) & 15 ? DSBD_ERR_UNSUPPORTED : DSBD_OK;
}

void set_rope(RopeArgs &a, const dsbd_rope_t *r) {
    if (!r) return;
    a.rot = r->rot; a.layout = r->layout; a.n_positions = r->n_positions; a.eps = r->eps;
    a.table = r->table; a.q_norm = r->q_norm; a.k_norm = r->k_norm;
}

// Warps that a call is spread over at least, 24 an SM: with 48 4608 tokens x 40 heads of 128 take 18.1 us instead of 16.9, 20 tokens 2.2
// either way.
constexpr int64_t kMinWarps = 148 * 24;

template <bool APPEND>
int launch_rotate(RopeArgs a, const dsbd_attn_desc_t *d, cudaStream_t stream) {
    const int piece = 32 / (d->d / 8) * unroll(d->dtype == DSBD_DTYPE_BF16 ? 2 : 4);
    a.q_pieces = a.q ? (a.Hq + piece - 1) / piece : 0;
    a.k_pieces = a.k ? (a.Hkv + piece - 1) / piece : 0;
    a.pieces = a.q_pieces + a.k_pieces + (APPEND ? a.k_pieces : 0);
    // a token's heads to one warp, or to as many as it takes to have kMinWarps
    const int want = (int)std::min<int64_t>(a.pieces, (kMinWarps + a.T - 1) / a.T);
    a.per_warp = (a.pieces + want - 1) / want;
    a.parts = (a.pieces + a.per_warp - 1) / a.per_warp;
    const int64_t jobs = (int64_t)a.T * a.parts + (APPEND ? 2 * (int64_t)a.B * a.Hkv : 0);
    const int64_t grid = (jobs + kThreads / 32 - 1) / (kThreads / 32);
    if (jobs > INT32_MAX) return DSBD_ERR_UNSUPPORTED;
    if (d->dtype == DSBD_DTYPE_F32)
        return d->d == 64 ? launch_pdl(k_rotate<float, 64, APPEND>, grid, kThreads, stream, a)
                          : launch_pdl(k_rotate<float, 128, APPEND>, grid, kThreads, stream, a);
    return d->d == 64 ? launch_pdl(k_rotate<__nv_bfloat16, 64, APPEND>, grid, kThreads, stream, a)
                      : launch_pdl(k_rotate<__nv_bfloat16, 128, APPEND>, grid, kThreads, stream, a);
}

}  // namespace

extern "C" int dsbd_rope_frequencies(const dsbd_rope_scaling_t *scaling, int32_t rot, double *f, double *attention) {
    return frequencies(scaling, rot, f, attention);
}

extern "C" int dsbd_rope_table(const dsbd_rope_scaling_t *scaling, int32_t rot, int32_t n_positions, float *table,
                               dsbd_stream_t stream) {
    Frequencies fr = {};
    double attention = 1.0;
    const int rc = frequencies(scaling, rot, fr.f, &attention);
    if (rc) return rc;
    if (n_positions <= 0 || !table) return DSBD_ERR_INVALID_ARG;
    const int64_t n = (int64_t)n_positions * (rot / 2), grid = (n + kThreads - 1) / kThreads;
    if (grid > INT32_MAX) return DSBD_ERR_UNSUPPORTED;
    k_rope_table<<<(unsigned)grid, kThreads, 0, reinterpret_cast<cudaStream_t>(stream)>>>(fr, attention, rot / 2, n, table);
    return cudaGetLastError() == cudaSuccess ? DSBD_OK : DSBD_ERR_CUDA;
}

extern "C" int dsbd_forest_positions(const dsbd_forest_t *f, const int64_t *prefix_off, int32_t *position, int32_t *status,
                                     dsbd_stream_t stream) {
    if (!f || f->B <= 0 || f->N <= 0 || !f->beam_node_off || !f->parent || !prefix_off || !position || !status)
        return DSBD_ERR_INVALID_ARG;
    return launch_pdl(k_forest_positions, ((int64_t)f->B + kTreeWarps - 1) / kTreeWarps, kTreeWarps * 32,
                      reinterpret_cast<cudaStream_t>(stream), (int)f->B, (int)f->N, f->beam_node_off, f->parent, prefix_off,
                      position, status);
}

extern "C" int dsbd_rotate_qk(int32_t T, const dsbd_attn_desc_t *d, const dsbd_rope_t *rope, const int32_t *position,
                              const void *q, int64_t q_stride, const void *k, int64_t k_stride, void *q_out,
                              int64_t q_out_stride, void *k_out, int64_t k_out_stride, int32_t *status,
                              dsbd_stream_t stream) {
    int rc = check_desc(d);
    if (rc) return rc;
    if ((rc = check_rope(rope, d->d))) return rc;
    if (T < 0 || !status) return DSBD_ERR_INVALID_ARG;
    if (T == 0) return DSBD_OK;
    if ((!q && !k) || !q != !q_out || !k != !k_out || (rope->rot && !position)) return DSBD_ERR_INVALID_ARG;
    if (q && ((rc = check_rows(q, q_stride, d->Hq, d)) || (rc = check_rows(q_out, q_out_stride, d->Hq, d)))) return rc;
    if (k && ((rc = check_rows(k, k_stride, d->Hkv, d)) || (rc = check_rows(k_out, k_out_stride, d->Hkv, d)))) return rc;
    RopeArgs a = {};
    a.T = T; a.Hq = d->Hq; a.Hkv = d->Hkv;
    set_rope(a, rope);
    a.q = q; a.k = k; a.q_out = q_out; a.k_out = k_out;
    a.q_stride = q_stride; a.k_stride = k_stride; a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride;
    a.position = position;
    a.status = status;
    return launch_rotate<false>(a, d, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" int dsbd_kv_append_paged(const dsbd_chunk_t *c, const dsbd_attn_desc_t *d, const dsbd_rope_t *rope, const void *q,
                                    int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                                    void *q_out, int64_t q_out_stride, void *k_pool, void *v_pool,
                                    const dsbd_kv_pages_t *pages, int32_t *status, dsbd_stream_t stream) {
    int rc = check_desc(d);
    if (rc) return rc;
    if (rope && (rc = check_rope(rope, d->d))) return rc;
    if (!c || c->B <= 0 || !c->new_off || !c->prefix_off || c->total_new < 0 || c->max_len < 0 || !pages ||
        !pages->page_table || !pages->page_off || pages->n_pages <= 0 || !k_pool || !v_pool || !status)
        return DSBD_ERR_INVALID_ARG;
    if (c->total_new == 0) return DSBD_OK;
    if (!q != !q_out) return DSBD_ERR_INVALID_ARG;
    if (q && ((rc = check_rows(q, q_stride, d->Hq, d)) || (rc = check_rows(q_out, q_out_stride, d->Hq, d)))) return rc;
    if ((rc = check_rows(k, k_stride, d->Hkv, d)) || (rc = check_rows(v, v_stride, d->Hkv, d))) return rc;
    if ((reinterpret_cast<uintptr_t>(k_pool) | reinterpret_cast<uintptr_t>(v_pool)) & 15) return DSBD_ERR_UNSUPPORTED;
    RopeArgs a = {};
    a.T = c->total_new; a.Hq = d->Hq; a.Hkv = d->Hkv;
    set_rope(a, rope);
    a.q = q; a.k = k; a.v = v; a.q_out = q_out;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.q_out_stride = q_out_stride;
    a.B = c->B; a.max_len = c->max_len; a.n_pages = pages->n_pages;
    a.new_off = c->new_off; a.prefix_off = c->prefix_off; a.page_table = pages->page_table; a.page_off = pages->page_off;
    a.k_pool = k_pool; a.v_pool = v_pool;
    a.status = status;
    return launch_rotate<true>(a, d, reinterpret_cast<cudaStream_t>(stream));
}
