// Attention of a chunk of new tokens over the paged cache that holds them, bf16, heads of 64 and 128, on the
// 5th-generation tensor cores (tcgen05 + TMEM + TMA).
//
//   out[i, h] = sum_j softmax_j(scale q[i, h] . K_j) V_j   over the positions j = 0 .. L_b + i of token i's sequence.
//
// Work unit = (sequence, KV head, block of tokens): the query rows of the block that map to this KV head (row = token *
// group + head) against the pages from the first to the block's last token, in tiles of 128 tokens (two pages).  A CTA
// has two row tiles of 128 rows, X = 0 and 1, each with a softmax warpgroup (a thread to a row, so maximum and sum of a row
// are one thread's), 128 columns of S in TMEM (the weights P, bf16, overwrite their first half) and its accumulators O:
//   S_X = Q_X K^T   (M = 128 rows, N = 128 tokens, K = d)    both operands K-major in shared memory
//   O_X += P_X V    (M = 128 rows, N = d, K = 128 tokens)    P from TMEM, V MN-major in shared memory
// While one group works on its S, the tensor cores work for the other: the products of X = 0 and 1 alternate.
//   wide   more than 128 rows: the tiles hold different rows, every K and V tile serves both.
//   narrow up to 128 rows (few tokens: single ones, ends of prompts): both tiles hold the same rows, X takes the K and V
//          tiles of its parity, and X = 0's group joins the two results at the end.  (The time of these units is the
//          cache's bytes; what counts is that the next copies are always on their way.)
// One warp issues the copies (K and V tiles through one ring of slots in the order in which they are used, the query rows),
// one the products.  Both run converged with one lane's predicate on the instructions.
//
// Masks: a unit ends with the tile of its block's last token; in the last tiles a row sees the tokens up to its own.  V rows
// behind the block's last token are cleared in shared memory, so that nothing in the pages behind it counts.
// A row's reference is its running maximum, moved only when a logit exceeds it by more than 2^8; P is rounded to bf16 (the
// operand type of V) and the row sum adds the rounded weights, so that a heavy weight's rounding cancels.
//
// Work split: the tiles of all units form one sequence (sequence, KV head, block), cut into equal runs, one per CTA; a unit
// that straddles a cut leaves partial results that k_chunk_merge joins.  Few short units are taken whole, one a CTA.  Every
// CTA finds its run with one scan over the sequences; there is no plan kernel.
//
// Every mbarrier wait is bounded; on a time-out the kernel records DSBD_DEV_TIMEOUT, lets its copies and products land,
// frees its TMEM and returns.
#include <math.h>

#include <algorithm>

#include "dsbd_tc.cuh"

using namespace dsbd;

namespace {

constexpr int kTile = 128;                           // tokens of a tile, rows of a row tile
constexpr int kPages = kTile / kBN;                  // pages of a tile
constexpr int kThreads = 384;                        // two softmax warpgroups, one with producer and issuer
constexpr int kWarpTma = 8, kWarpMma = 9;
constexpr uint32_t kHalf = kTile * 128;              // bytes of 64 columns of a tile
constexpr uint32_t kTmemCols = 512, kColS = 0, kColO = 256;
constexpr float kMoveRef = 8.f;
// Registers: launched with 168 a thread (64512); 256 softmax threads of 232 and 128 others of 40 are as many.
constexpr int kSoftmaxRegs = 232, kOtherRegs = 40;
static_assert(kSoftmaxRegs * 256 + kOtherRegs * 128 <= 168 * kThreads, "no more than at launch");
#ifdef DSBD_TEST_WAIT_TIMEOUT
constexpr uint32_t kWaitTries = 250;                 // test build: see dsbd_attention_tr.cu
#else
constexpr uint32_t kWaitTries = 500000;              // about two seconds: a try is suspended for 4 us
#endif

template <int D>
struct Shape {
    static constexpr int kHalves = D / 64;
    static constexpr uint32_t kSlot = kHalves * kHalf;          // a K or V tile; the rows of a row tile
    static constexpr int kSlots = D == 128 ? 5 : 8;
    static constexpr uint32_t kSmem = 1024 + 2 * kSlot + kSlots * kSlot;
};

struct ChunkArgs {
    int B, Hq, Hkv, group, T;
    int tile_tokens, block_tokens;                   // tokens of a row tile (128 / group) and of a block (two)
    int box_tokens;                                  // of a query box
    int whole;                                       // a unit a CTA, nothing is cut
    int unit_cost;                                   // what a unit costs beside its tokens, in tokens
    float scale_log2;
    int64_t max_len, n_pages, min_run;               // min_run: smallest run, in cost
    const int32_t *new_off, *page_table;
    const int64_t *prefix_off, *page_off;
    __nv_bfloat16 *out;
    int32_t *status;
    struct CutRec *recs;                             // [grid]
    float *partial;                                  // [2 * grid][256][D + 2]: reference, row sum, O
};

// A place in the work: unit (b, g, q) and a tile of it.
struct Pos { int b, g, q, t; };
__device__ __forceinline__ bool before(const Pos &x, const Pos &y) {
    if (x.b != y.b) return x.b < y.b;
    if (x.g != y.g) return x.g < y.g;
    if (x.q != y.q) return x.q < y.q;
    return x.t < y.t;
}

// What a run left for the merge.  tail: a unit that it began and did not end; head: how it went on with one that an earlier
// run began (0 not at all, 1 not to its end, 2 to its end).
struct CutRec { int tail, head, b, g, q, pad[3]; };

struct Seq { int n, first; int64_t L; };
__device__ __forceinline__ Seq seq_of(const ChunkArgs &a, int b, bool tell) {
    Seq s;
    s.first = a.new_off[b];
    const int end = a.new_off[b + 1];
    s.L = a.prefix_off[b + 1] - a.prefix_off[b];
    s.n = end - s.first;
    if (s.first < 0 || end < s.first || end > a.T || s.L < 0 || s.L > a.max_len || s.L + s.n > a.max_len) {
        s.n = 0;
        if (tell) report(a.status, DSBD_DEV_BAD_CHUNK);
    }
    return s;
}
__device__ __forceinline__ int blocks_of(const ChunkArgs &a, int n) { return (n + a.block_tokens - 1) / a.block_tokens; }
// Cost of the first q blocks of one head of a sequence.
__device__ __forceinline__ int64_t cost_before(const ChunkArgs &a, const Seq &s, int q) {
    const int64_t full = (int64_t)q * (s.L + a.unit_cost) + (int64_t)a.block_tokens * ((int64_t)q * (q + 1) / 2);
    return q < blocks_of(a, s.n) || q == 0 ? full : full - ((int64_t)q * a.block_tokens - s.n);
}
__device__ __forceinline__ int64_t head_cost(const ChunkArgs &a, const Seq &s) {
    const int nq = blocks_of(a, s.n);
    return a.whole ? nq : cost_before(a, s, nq);
}

struct Unit {
    int first, n;                                    // rows of the sequence
    int64_t L;
    int i0, tokens;                                  // the block's first token and number of tokens
    int64_t end;                                     // tokens that the block's last one sees
    int nt;
    bool wide;
};
__device__ __forceinline__ Unit unit_of(const ChunkArgs &a, const Seq &s, int q) {
    Unit u;
    u.first = s.first; u.n = s.n; u.L = s.L;
    u.i0 = q * a.block_tokens;
    u.tokens = min(a.block_tokens, s.n - u.i0);
    u.end = s.L + u.i0 + u.tokens;
    u.nt = (int)((u.end + kTile - 1) / kTile);
    u.wide = u.tokens > a.tile_tokens;
    return u;
}

// Walks a run: the parts of units from `at` to `end`.
struct Walk {
    Pos at, end;
    Seq s;
    int nq;
    __device__ __forceinline__ void start(const ChunkArgs &a, const Pos &p0, const Pos &p1) {
        at = p0; end = p1;
        if (before(at, end)) { s = seq_of(a, at.b, false); nq = blocks_of(a, s.n); }
    }
    __device__ __forceinline__ bool more() const { return before(at, end); }
    __device__ __forceinline__ int last_tile(const Unit &u) const {
        return at.b == end.b && at.g == end.g && at.q == end.q ? min(end.t, u.nt) : u.nt;
    }
    __device__ __forceinline__ void next(const ChunkArgs &a, int heads) {
        at.t = 0;
        if (++at.q < nq) return;
        at.q = 0;
        if (++at.g < heads) return;
        at.g = 0;
        do {
            ++at.b;
            if (!before(at, end)) return;
            s = seq_of(a, at.b, false);
        } while (s.n == 0);
        nq = blocks_of(a, s.n);
    }
};

// Where the K and V tiles of a part of nt tiles lie in the order of the ring: `ahead` K tiles first (1 wide, 2 narrow),
// then V tile i and K tile i + ahead in turn.
__device__ __forceinline__ uint32_t seq_k(int i, int ahead) { return i < ahead ? i : 2 * i - ahead + 1; }
__device__ __forceinline__ uint32_t seq_v(int i, int nt, int ahead) {
    const int first = min(ahead, nt);
    return first + i + min(i, nt - first);
}

struct Shared {
    unsigned long long full[8], empty[8], s_full[2], p_full[2], o_full[2], q_full, q_empty, b_done, b_free, drain;
    uint32_t tmem_base;
    int abort;
    Pos start, end;
    int64_t scan[kThreads / 32], mine[2];
    int found_b[2];
    float ml[2][kTile];                              // reference and row sum of the narrow units' second half
};

__device__ __forceinline__ bool warp_wait(void *bar, uint32_t parity, Shared *sh) {
    bool ok = true;
#pragma unroll 1
    for (uint32_t i = 0; !mbar_try(bar, parity); ++i)
        if (i == kWaitTries || *reinterpret_cast<volatile int *>(&sh->abort)) {
            *reinterpret_cast<volatile int *>(&sh->abort) = 1;
            ok = false;
            break;
        }
    return __all_sync(kFull, ok);
}

struct F2 { float x, y; };
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
    F2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// The CTA's run: all threads.  Returns through sh.start, sh.end; the sequences' facts are checked here, once a launch.
__device__ void find_run(const ChunkArgs &a, Shared &sh) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (a.B + kThreads - 1) / kThreads, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
    int64_t sum = 0;
    for (int b = b0; b < b1; ++b) sum += head_cost(a, seq_of(a, b, blockIdx.x == 0)) * a.Hkv;
    int64_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(kFull, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) sh.scan[warp] = incl;
    if (tid < 2) sh.found_b[tid] = -1;
    __syncthreads();
    int64_t base = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) base += sh.scan[w];
        total += sh.scan[w];
    }
    const int64_t hi = base + incl, lo = hi - sum;
    // the cuts: equal runs of at least min_run
    int64_t runs = a.whole ? total : total / a.min_run;
    runs = runs < 1 ? 1 : runs > (int64_t)gridDim.x ? (int64_t)gridDim.x : runs;
    int64_t cut[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int64_t c = (int64_t)blockIdx.x + k;
        cut[k] = c >= runs ? total : a.whole ? c : total / runs * c + total % runs * c / runs;
        if (cut[k] >= lo && cut[k] < hi) {
            int64_t x = lo;
            for (int b = b0; b < b1; ++b) {
                const Seq s = seq_of(a, b, false);
                const int64_t hc = head_cost(a, s), c_b = hc * a.Hkv;
                if (cut[k] >= x + c_b) { x += c_b; continue; }
                const int64_t rem = cut[k] - x;
                Pos p;
                p.b = b;
                p.g = (int)(rem / hc);
                int64_t in = rem - p.g * hc;
                const int nq = blocks_of(a, s.n);
                if (a.whole) {
                    p.q = (int)in; p.t = 0;
                } else {
                    // largest q with cost_before(q) <= in: the root of a quadratic, put right by steps
                    const double h = (double)(s.L + a.unit_cost) / a.block_tokens + 0.5;
                    int q = (int)(sqrt(h * h + 2.0 * (double)in / a.block_tokens) - h);
                    q = max(0, min(q, nq - 1));
                    while (q > 0 && cost_before(a, s, q) > in) --q;
                    while (q + 1 < nq && cost_before(a, s, q + 1) <= in) ++q;
                    p.q = q;
                    in -= cost_before(a, s, q) + a.unit_cost;
                    p.t = in > 0 ? (int)(in / kTile) : 0;
                }
                if (k == 0) sh.start = p; else sh.end = p;
                sh.found_b[k] = b;
                break;
            }
        }
    }
    __syncthreads();
    if (tid == 0) {
        const Pos over = {a.B, 0, 0, 0};
        if (sh.found_b[0] < 0) sh.start = over;
        if (sh.found_b[1] < 0) sh.end = over;
    }
    __syncthreads();
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
k_chunk_attn(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
             const __grid_constant__ CUtensorMap map_q, ChunkArgs a) {
    using S = Shape<D>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);    // swizzled operands
    unsigned char *q_s = smem, *ring = smem + 2 * S::kSlot;
    __shared__ Shared sh;
    const int warp = __shfl_sync(kFull, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kSlots; ++s) { mbar_init(&sh.full[s], 1); mbar_init(&sh.empty[s], 1); }
        for (int x = 0; x < 2; ++x) { mbar_init(&sh.s_full[x], 1); mbar_init(&sh.p_full[x], 4); mbar_init(&sh.o_full[x], 1); }
        mbar_init(&sh.q_full, 1);
        mbar_init(&sh.q_empty, 1);
        mbar_init(&sh.b_done, 4);
        mbar_init(&sh.b_free, 4);
        mbar_init(&sh.drain, 1);
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kWarpMma) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)),
                     "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    find_run(a, sh);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(&sh.tmem_base);

    if (threadIdx.x == 0 && a.recs) {
        CutRec r = {};
        const Pos p0 = sh.start, p1 = sh.end;
        const bool same = p0.b == p1.b && p0.g == p1.g && p0.q == p1.q;
        r.tail = p1.t > 0 && (!same || p0.t == 0);
        r.head = p0.t == 0 ? 0 : !same ? 2 : p1.t > p0.t ? 1 : 0;
        r.b = p1.b; r.g = p1.g; r.q = p1.q;
        a.recs[blockIdx.x] = r;
    }

    if (warp >= 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    Walk w;
    w.start(a, sh.start, sh.end);
    if (warp == kWarpTma) {
        // ------------------------------------------------------------ copies
        uint32_t seq = 0, part = 0;
        bool ok = true;
        for (; ok && w.more(); w.next(a, a.Hkv)) {
            const Unit u = unit_of(a, w.s, w.at.q);
            const int t0 = w.at.t, nt = w.last_tile(u) - t0, g = w.at.g;
            if (nt <= 0) continue;
            const int ahead = u.wide ? 1 : 2;
            if (part > 0) ok = warp_wait(&sh.q_empty, (part - 1) & 1, &sh);
            if (!ok) break;
            ++part;
            const bool on = lane == 0;
            const int tiles = u.wide ? 2 : 1;
            mbar_expect_tx_if(on, &sh.q_full, (uint32_t)(tiles * a.box_tokens * a.group * D * 2));
            for (int x = 0; x < tiles; ++x)
#pragma unroll
                for (int h = 0; h < S::kHalves; ++h)
                    tma_load_3d(on, smem_u32(q_s + x * S::kSlot + h * kHalf), &map_q, h * 64, g * a.group,
                                u.first + u.i0 + x * a.tile_tokens, &sh.q_full);
            // K and V of a sequence with one block of rows pass once
            uint64_t policy;
            if (w.nq == 1) asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
            else asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
            // page ids of the part, 32 in a warp's registers
            const int64_t table0 = a.page_off[w.at.b], n_table = a.page_off[w.at.b + 1] - table0;
            const int p_end = (int)((u.end + kBN - 1) / kBN);            // pages of the unit
            int base = t0 * kPages;
            auto fetch = [&](int from) -> int {
                const int p = from + lane;
                int id = -1;
                if (p < p_end && p < (t0 + nt) * kPages) {
                    if (p < n_table) {
                        id = a.page_table[table0 + p];
                        if (id < 0 || id >= a.n_pages) { report(a.status, DSBD_DEV_BAD_CHUNK); id = -1; }
                    } else {
                        report(a.status, DSBD_DEV_CAPACITY);
                    }
                }
                return id;
            };
            int ids_k = fetch(base), ids_v = ids_k, base_k = base, base_v = base;
            auto copy = [&](const CUtensorMap *map, int tile, int &ids, int &at) {
                const int p = (t0 + tile) * kPages;
                if (p >= at + 32) { at = p; ids = fetch(p); }
                const int s = seq % S::kSlots;
                if (!warp_wait(&sh.empty[s], ((seq / S::kSlots) & 1) ^ 1, &sh)) { ok = false; return; }
                const int boxes = min(kPages, p_end - p);
                mbar_expect_tx_if(on, &sh.full[s], (uint32_t)boxes * kBN * D * 2);
                const uint32_t dst = smem_u32(ring + s * S::kSlot);
#ifdef DSBD_TEST_WAIT_TIMEOUT
                const bool there = !(seq == 1 && blockIdx.x == 0);       // the bytes this barrier expects never come
#else
                const bool there = true;
#endif
                for (int k = 0; k < boxes; ++k) {
                    const int id = __shfl_sync(kFull, ids, p + k - at);
                    const int y = id < 0 ? INT32_MAX - 2 * kBN : (id * a.Hkv + g) * kBN;      // (past the pool: zeros)
#pragma unroll
                    for (int h = 0; h < S::kHalves; ++h)
                        tma_load_2d_hint(on && there, dst + h * kHalf + k * (kBN * 128), map, h * 64, y, &sh.full[s], policy);
                }
                ++seq;
            };
            for (int i = 0; i < min(ahead, nt) && ok; ++i) copy(&map_k, i, ids_k, base_k);
            for (int i = 0; i < nt && ok; ++i) {
                copy(&map_v, i, ids_v, base_v);
                if (ok && i + ahead < nt) copy(&map_k, i + ahead, ids_k, base_k);
            }
        }
        if (!ok) {
            // let the copies already issued land before the CTA goes away
            for (uint32_t k = 0; k < (uint32_t)S::kSlots && k < seq; ++k) {
                const uint32_t t = seq - 1 - k;
                for (uint32_t i = 0; i < kWaitTries && !mbar_try(&sh.full[t % S::kSlots], (t / S::kSlots) & 1); ++i) {}
            }
            if (part > 0)
                for (uint32_t i = 0; i < kWaitTries && !mbar_try(&sh.q_full, (part - 1) & 1); ++i) {}
        }
    } else if (warp == kWarpMma) {
        // ------------------------------------------------------------ products
        const bool on = lane == 0;
        constexpr uint32_t idesc_s = instr_desc(kTile, kTile, 0, 0);
        constexpr uint32_t idesc_o = instr_desc(kTile, D, 0, 1);
        uint32_t base = 0, part = 0, np[2] = {0, 0};
        bool ok = true;
        auto slot_wait = [&](uint32_t seq) -> uint32_t {
            const uint32_t s = seq % S::kSlots;
            ok = warp_wait(&sh.full[s], (seq / S::kSlots) & 1, &sh);
            return s;
        };
        for (; ok && w.more(); w.next(a, a.Hkv)) {
            const Unit u = unit_of(a, w.s, w.at.q);
            const int nt = w.last_tile(u) - w.at.t;
            if (nt <= 0) continue;
            const int ahead = u.wide ? 1 : 2, steps = u.wide ? 2 * nt : nt;
            int left = steps;                        // S products to come
            ok = warp_wait(&sh.q_full, part & 1, &sh);
            auto product_s = [&](int x, int i) {
                const uint32_t s = slot_wait(base + seq_k(i, ahead));
                if (!ok) return;
                tc_fence_after();
                const uint64_t qd = desc_k_major(smem_u32(q_s + (u.wide ? x : 0) * S::kSlot));
                const uint64_t kd = desc_k_major(smem_u32(ring + s * S::kSlot));
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint64_t at = (uint64_t)((ks / 4) * (kHalf >> 4) + (ks % 4) * 2);
                    mma_ss(on, tmem + kColS + x * kTile, qd + at, kd + at, idesc_s, ks > 0);
                }
                tc_commit(on, &sh.s_full[x]);
                if (!u.wide || x == 1) tc_commit(on, &sh.empty[s]);
                if (--left == 0) tc_commit(on, &sh.q_empty);
            };
            for (int x = 0; x < min(2, steps) && ok; ++x) product_s(x, u.wide ? 0 : x);
            for (int st = 0; st < steps && ok; ++st) {
                const int x = st & 1, i = u.wide ? st >> 1 : st;
                const uint32_t s = slot_wait(base + seq_v(i, nt, ahead));
                if (!ok) break;
                ok = warp_wait(&sh.p_full[x], np[x] & 1, &sh);
                if (!ok) break;
                ++np[x];
                tc_fence_after();
                const uint64_t vd = desc_mn_major(smem_u32(ring + s * S::kSlot), kHalf);
                const bool fresh = u.wide ? i == 0 : i < 2;
#pragma unroll
                for (int ks = 0; ks < kTile / 16; ++ks)
                    mma_ts(on, tmem + kColO + x * D, tmem + kColS + x * kTile + ks * 8, vd + (uint64_t)(ks * ((16 * 128) >> 4)),
                           idesc_o, (!fresh || ks > 0) ? 1u : 0u);
                if (!u.wide || x == 1) tc_commit(on, &sh.empty[s]);
                if (i + ahead < nt) product_s(x, i + ahead);
                else tc_commit(on, &sh.o_full[x]);
            }
            base += 2 * nt;
            ++part;
        }
        if (!ok) {
            tc_commit(on, &sh.drain);
            uint32_t i = 0;
            while (!__all_sync(kFull, mbar_try(&sh.drain, 0)) && i < kWaitTries) ++i;
        }
    } else if (warp < 8) {
        // ------------------------------------------------------------ softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        const int x = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_addr = tmem + lanes + kColS + x * kTile, o_addr = tmem + lanes + kColO + x * D;
        const int token = row / a.group, head = row - token * a.group;
        uint32_t base = 0, ns = 0, no = 0, narrow = 0;
        bool ok = true;
        for (; ok && w.more(); w.next(a, a.Hkv)) {
            const Unit u = unit_of(a, w.s, w.at.q);
            const int t0 = w.at.t, nt = w.last_tile(u) - t0;
            if (nt <= 0) continue;
            const int ahead = u.wide ? 1 : 2;
            const int i0 = u.i0 + (u.wide ? x * a.tile_tokens : 0);          // the row tile's first token
            const int left = min(a.tile_tokens, u.n - i0);                   // its tokens
            const bool active = token < left;
            const bool work = (warp & 3) * 32 < left * a.group;              // some row of the warp
            const int64_t sees = u.L + i0 + token + 1;                       // tokens the row sees
            const int64_t all_see = u.L + i0 + 1;                            // every row of the tile
            const int step = u.wide ? 1 : 2, mine = u.wide ? nt : (nt - x + 1) / 2;
            float m_ref = -INFINITY, l = 0.f;
            for (int i = u.wide ? 0 : x; i < nt; i += step) {
                ok = warp_wait(&sh.s_full[x], ns & 1, &sh);
                if (!ok) break;
                ++ns;
                tc_fence_after();
                const int64_t tok0 = (int64_t)(t0 + i) * kTile;
                if (work) {
                    uint32_t sv[4][32];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld32(s_addr + c * 32, sv[c]);
                    tmem_wait_ld();
                    if (tok0 + kTile > all_see) {
                        const int lim = (int)min((int64_t)kTile, max((int64_t)0, sees - tok0));
#pragma unroll
                        for (int c = 0; c < kTile; ++c)
                            if (c >= lim) sv[c >> 5][c & 31] = 0xff800000u;      // -inf: weight 0
                    }
                    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < kTile; c += 2)
                        m4[(c >> 1) & 3] = max3(m4[(c >> 1) & 3], __uint_as_float(sv[c >> 5][c & 31]), __uint_as_float(sv[c >> 5][(c & 31) + 1]));
                    const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * a.scale_log2;    // scale > 0
                    const bool need = mx > m_ref + kMoveRef;
                    if (__any_sync(kFull, need)) {
                        // (the tile's S product was issued behind the previous O product, so that one has landed)
                        const float m_new = need ? mx : m_ref;
                        const float f = m_ref == -INFINITY ? 0.f : exp2f(m_ref - m_new);
                        l *= f;
                        if (i >= step) {
#pragma unroll 1
                            for (int c = 0; c < D; c += 32) {
                                uint32_t ov[32];
                                tmem_ld32(o_addr + c, ov);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 32; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * f);
                                tmem_st32(o_addr + c, ov);
                            }
                        }
                        m_ref = m_new;
                    }
                    const float neg = m_ref == -INFINITY ? 0.f : -m_ref;
                    F2 l2[2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t pv[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const int at = c * 64 + 2 * e;
                            const F2 z = fma2(F2{__uint_as_float(sv[at >> 5][at & 31]), __uint_as_float(sv[at >> 5][(at & 31) + 1])},
                                              F2{a.scale_log2, a.scale_log2}, F2{neg, neg});
                            pv[e] = pack_bf16(ex2_ftz(z.x), ex2_ftz(z.y));
                            l2[e & 1] = add2(l2[e & 1], F2{bf16_lo(pv[e]), bf16_hi(pv[e])});
                        }
                        tmem_st32(s_addr + c * 32, pv);
                    }
                    l += (l2[0].x + l2[0].y) + (l2[1].x + l2[1].y);
                    tmem_wait_st();
                }
                // what lies behind the block's last token has weight zero: its values become zeros
                if (tok0 + kTile > u.end && (x == 0 || !u.wide)) {
                    const uint32_t sv = base + seq_v(i, nt, ahead), s = sv % S::kSlots;
                    ok = warp_wait(&sh.full[s], (sv / S::kSlots) & 1, &sh);
                    if (!ok) break;
                    const int valid = (int)(u.end - tok0);
                    if (row >= valid) {
#pragma unroll
                        for (int h = 0; h < S::kHalves; ++h) {
                            uint4 *line = reinterpret_cast<uint4 *>(ring + s * S::kSlot + h * kHalf + row * 128);
#pragma unroll
                            for (int e = 0; e < 8; ++e) line[e] = make_uint4(0, 0, 0, 0);
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                // (the accumulators of a narrow unit's second half are free once the first group has read them)
                if (x == 1 && i < step && narrow > 0) {
                    ok = warp_wait(&sh.b_free, (narrow - 1) & 1, &sh);
                    if (!ok) break;
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.p_full[x]);
            }
            if (!ok) break;
            base += 2 * nt;
            if (mine > 0) {
                ok = warp_wait(&sh.o_full[x], no & 1, &sh);
                if (!ok) break;
                ++no;
                tc_fence_after();
            }
            // ---- the end of the unit, or of its part
            float fo = 1.f, fb = 0.f;                        // factors of this tile's O and of the second half's
            bool second = false;
            if (!u.wide) {
                if (x == 1) {
                    // (the first group has read those of the narrow unit before)
                    if (narrow > 0) ok = warp_wait(&sh.b_free, (narrow - 1) & 1, &sh);
                    if (!ok) break;
                    sh.ml[0][row] = m_ref;
                    sh.ml[1][row] = l;
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.b_done);
                    ++narrow;
                    continue;
                }
                ok = warp_wait(&sh.b_done, narrow & 1, &sh);
                if (!ok) break;
                tc_fence_after();
                second = nt > 1;
                const float mb = sh.ml[0][row], lb = sh.ml[1][row];
                const float m = fmaxf(m_ref, mb);
                fo = m_ref == -INFINITY ? 0.f : exp2f(m_ref - m);
                fb = mb == -INFINITY ? 0.f : exp2f(mb - m);
                l = l * fo + lb * fb;
                m_ref = m;
            }
            const bool is_whole = t0 == 0 && nt == u.nt;
            if (work) {
                const int r = (u.wide ? x * a.tile_tokens * a.group : 0) + row;
                float *part = nullptr;
                __nv_bfloat16 *dst = a.out + ((int64_t)(u.first + i0 + token) * a.Hq + w.at.g * a.group + head) * D;
                if (is_whole) {
                    const float inv = 1.f / l;
                    fo *= inv; fb *= inv;
                } else {
                    part = a.partial + ((2 * (int64_t)blockIdx.x + (t0 == 0 ? 1 : 0)) * 256 + r) * (D + 2);
                    if (active) { part[0] = m_ref; part[1] = l; }
                }
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t ov[32], ow[32];
                    tmem_ld32(o_addr + c, ov);
                    if (second) tmem_ld32(o_addr + D + c, ow);
                    tmem_wait_ld();
                    float o[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        o[e] = __uint_as_float(ov[e]) * fo;
                        if (second) o[e] = fmaf(__uint_as_float(ow[e]), fb, o[e]);
                    }
                    if (active && is_whole) {
#pragma unroll
                        for (int e = 0; e < 32; e += 8)
                            *reinterpret_cast<uint4 *>(dst + c + e) =
                                make_uint4(pack_bf16(o[e], o[e + 1]), pack_bf16(o[e + 2], o[e + 3]),
                                           pack_bf16(o[e + 4], o[e + 5]), pack_bf16(o[e + 6], o[e + 7]));
                    } else if (active) {
#pragma unroll
                        for (int e = 0; e < 32; e += 2) *reinterpret_cast<float2 *>(part + 2 + c + e) = make_float2(o[e], o[e + 1]);
                    }
                    __syncwarp();
                }
            }
            tc_fence_before();
            if (!u.wide) {
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.b_free);
                ++narrow;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *reinterpret_cast<volatile int *>(&sh.abort)) report(a.status, DSBD_DEV_TIMEOUT);
    if (warp == kWarpMma) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

// Joins the parts of cut units: block (i, y) takes the unit that run i began and did not end, a warp to a row;
// out = sum_p O_p 2^(m_p - m) / sum_p l_p 2^(m_p - m), the parts in the order of their runs.
constexpr int kMergeThreads = 256, kMergeRows = 4;                       // rows of a warp
template <int D>
__global__ void __launch_bounds__(kMergeThreads)
k_chunk_merge(ChunkArgs a, int runs) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int i0 = blockIdx.x, lane = threadIdx.x & 31;
    const CutRec rec = a.recs[i0];
    if (!rec.tail) return;
    const Seq s = seq_of(a, rec.b, false);
    const Unit u = unit_of(a, s, rec.q);
    const int rows = u.tokens * a.group;
    if ((int)blockIdx.y * (kMergeThreads / 32 * kMergeRows) >= rows) return;
    int last = i0;
    for (int h = 1; h == 1 && last + 1 < runs;) h = a.recs[++last].head;
    constexpr int kPer = D / 32;
    for (int k = 0; k < kMergeRows; ++k) {
        const int row = (blockIdx.y * kMergeRows + k) * (kMergeThreads / 32) + (threadIdx.x >> 5);
        if (row >= rows) return;
        auto part = [&](int i) { return a.partial + ((2 * (int64_t)i + (i == i0 ? 1 : 0)) * 256 + row) * (D + 2); };
        float m = -INFINITY;
        for (int i = i0; i <= last; ++i)
            if (i == i0 || a.recs[i].head) m = fmaxf(m, part(i)[0]);
        float l = 0.f, o[kPer] = {};
        for (int i = i0; i <= last; ++i) {
            if (i != i0 && !a.recs[i].head) continue;
            const float *src = part(i);
            if (src[0] == -INFINITY) continue;
            const float f = exp2f(src[0] - m);
            l += src[1] * f;
#pragma unroll
            for (int e = 0; e < kPer; e += 2) {
                const float2 v = *reinterpret_cast<const float2 *>(src + 2 + lane * kPer + e);
                o[e] += v.x * f; o[e + 1] += v.y * f;
            }
        }
        const float inv = 1.f / l;
        const int token = row / a.group, head = row - token * a.group;
        uint32_t *dst = reinterpret_cast<uint32_t *>(
            a.out + ((int64_t)(u.first + u.i0 + token) * a.Hq + rec.g * a.group + head) * D + lane * kPer);
#pragma unroll
        for (int e = 0; e < kPer; e += 2) dst[e / 2] = pack_bf16(o[e] * inv, o[e + 1] * inv);
    }
}

// Launch shape shared by the workspace query and the launch.
struct Plan { int grid, whole, block_rows; };
constexpr int64_t kWholeTiles = 12;                  // longest units that are taken whole
constexpr int64_t kMinRun = 4 * kTile;               // smallest run, in tokens

Plan make_plan(const dsbd_chunk_t *c, const dsbd_attn_desc_t *d) {
    Plan p = {};
    int dev = 0, sms = 148;
    if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    const int group = d->Hq / d->Hkv, block = 2 * (kTile / group);
    p.block_rows = (int)std::min<int64_t>(block, c->max_new) * group;
    // an upper bound of the units
    const int64_t units = (int64_t)d->Hkv * std::min<int64_t>(c->total_new, c->max_new <= block ? c->B : (int64_t)c->B + c->total_new / block);
    p.whole = units <= sms && c->max_len <= kWholeTiles * kTile;
    p.grid = p.whole ? (int)units : sms;
    return p;
}

int check(const dsbd_chunk_t *c, const dsbd_attn_desc_t *d) {
    if (!c || !d || c->B <= 0 || !c->new_off || !c->prefix_off || c->total_new < 0 || c->max_new < 0 || c->max_len < 0)
        return DSBD_ERR_INVALID_ARG;
    if (d->Hq <= 0 || d->Hkv <= 0 || d->Hq % d->Hkv || !(d->scale > 0.f) || !std::isfinite(d->scale)) return DSBD_ERR_INVALID_ARG;
    if (d->dtype != DSBD_DTYPE_BF16 || (d->d != 64 && d->d != 128) || d->Hq / d->Hkv > kTile) return DSBD_ERR_UNSUPPORTED;
    if (c->max_len > (int64_t)1 << 30) return DSBD_ERR_UNSUPPORTED;
    return DSBD_OK;
}

size_t workspace_of(const Plan &p, int d) {
    if (p.whole) return 256;
    return align_up(sizeof(CutRec) * (size_t)p.grid, 256) + align_up(sizeof(float) * 2 * (size_t)p.grid * 256 * (d + 2), 256);
}

template <int D>
int launch(const Plan &p, const CUtensorMap (&maps)[3], const ChunkArgs &a, cudaStream_t stream) {
    using S = Shape<D>;
    if (cudaFuncSetAttribute(k_chunk_attn<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem) != cudaSuccess)
        return DSBD_ERR_CUDA;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, k_chunk_attn<D>, maps[0], maps[1], maps[2], a) != cudaSuccess) return DSBD_ERR_CUDA;
    if (p.whole) return DSBD_OK;
    const int per = kMergeThreads / 32 * kMergeRows;
    cfg.gridDim = dim3((unsigned)p.grid, (unsigned)((p.block_rows + per - 1) / per));
    cfg.blockDim = dim3(kMergeThreads);
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, k_chunk_merge<D>, a, p.grid) == cudaSuccess ? DSBD_OK : DSBD_ERR_CUDA;
}

}  // namespace

extern "C" size_t dsbd_chunk_attention_paged_workspace(const dsbd_chunk_t *c, const dsbd_attn_desc_t *d) {
    if (check(c, d) != DSBD_OK) return 0;
    return c->total_new == 0 ? 256 : workspace_of(make_plan(c, d), d->d);
}

extern "C" int dsbd_chunk_attention_paged_launches(const dsbd_chunk_t *c, const dsbd_attn_desc_t *d) {
    if (check(c, d) != DSBD_OK || c->total_new == 0) return 0;
    return make_plan(c, d).whole ? 1 : 2;
}

extern "C" int dsbd_chunk_attention_paged(const dsbd_chunk_t *c, const dsbd_attn_desc_t *d, const void *q, const void *k_pool,
                                          const void *v_pool, const dsbd_kv_pages_t *pages, void *out, void *workspace,
                                          size_t workspace_bytes, int32_t *status, dsbd_stream_t stream_) {
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    const int rc = check(c, d);
    if (rc) return rc;
    if (c->total_new == 0) return DSBD_OK;
    if (!q || !k_pool || !v_pool || !out || out == q || !status || !pages || !pages->page_table || !pages->page_off || pages->n_pages <= 0)
        return DSBD_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k_pool) | reinterpret_cast<uintptr_t>(v_pool) |
         reinterpret_cast<uintptr_t>(out)) & 15)
        return DSBD_ERR_UNSUPPORTED;
    // row coordinates of the pools' maps are 32-bit (and one past them names no row)
    const int64_t rows = pages->n_pages * d->Hkv * kBN;
    if (pages->n_pages > INT32_MAX || rows > INT32_MAX - 4 * kBN) return DSBD_ERR_UNSUPPORTED;
    const Plan plan = make_plan(c, d);
    if (!workspace || workspace_bytes < workspace_of(plan, d->d)) return DSBD_ERR_WORKSPACE_TOO_SMALL;
    if (!plan.whole && (reinterpret_cast<uintptr_t>(workspace) & 255)) return DSBD_ERR_INVALID_ARG;
    ChunkArgs a = {};
    a.B = c->B; a.Hq = d->Hq; a.Hkv = d->Hkv; a.group = d->Hq / d->Hkv; a.T = c->total_new;
    a.tile_tokens = kTile / a.group;
    a.block_tokens = 2 * a.tile_tokens;
    a.box_tokens = std::min(a.tile_tokens, c->total_new);
    a.whole = plan.whole;
    a.unit_cost = kTile;
    a.min_run = kMinRun;
    a.scale_log2 = d->scale * 1.4426950408889634f;
    a.max_len = c->max_len; a.n_pages = pages->n_pages;
    a.new_off = c->new_off; a.prefix_off = c->prefix_off; a.page_table = pages->page_table; a.page_off = pages->page_off;
    a.out = static_cast<__nv_bfloat16 *>(out);
    a.status = status;
    if (!plan.whole) {
        a.recs = static_cast<CutRec *>(workspace);
        a.partial = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + align_up(sizeof(CutRec) * (size_t)plan.grid, 256));
    }
    CUtensorMap maps[3];
    const uint64_t D = (uint64_t)d->d;
    if (!make_map(&maps[0], k_pool, D, (uint64_t)rows, D * 2) || !make_map(&maps[1], v_pool, D, (uint64_t)rows, D * 2) ||
        !make_map_q(&maps[2], q, D, (uint64_t)d->Hq, (uint64_t)c->total_new, (uint32_t)a.group, (uint32_t)a.box_tokens))
        return DSBD_ERR_CUDA;
    return d->d == 64 ? launch<64>(plan, maps, a, stream) : launch<128>(plan, maps, a, stream);
}
