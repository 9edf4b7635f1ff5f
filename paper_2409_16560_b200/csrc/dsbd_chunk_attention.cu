// Attention of a chunk of new tokens over the paged cache that holds them, bf16, heads of 64 and 128, on the
// 5th-generation tensor cores (tcgen05 + TMEM + TMA).
//
//   out[i, h] = sum_j softmax_j(scale q[i, h] . K_j) V_j   over the positions j = 0 .. L_b + i of token i's sequence.
//
// Work unit = (sequence, KV head, block of tokens): the query rows of the block that map to this KV head (row = token *
// group + head) against the pages from the first to the block's last token, in tiles of a page (64 tokens).  A CTA has two row
// tiles of 128 rows, X = 0 and 1, each with a softmax warpgroup (a thread to a row, so maximum and sum of a row are one thread's),
// two buffers of 64 columns for S in TMEM (the weights P, bf16, overwrite the first half of theirs) and its accumulators O:
//   S_X = Q_X K^T   (M = 128 rows, N = 64 tokens, K = d)    both operands K-major in shared memory
//   O_X += P_X V    (M = 128 rows, N = d, K = 64 tokens)    P from TMEM, V MN-major in shared memory
// S runs two of a row tile's tiles ahead of O, so neither a softmax nor the tensor cores wait for the other's latency.  (Tiles of
// 128 tokens read less of Q but leave TMEM no second buffer: the chain from a row tile's P over O and S to its next softmax then
// took 3600 cycles for 128 tokens, two tiles of 64 take 3100.)
//   wide   more than 128 rows: the row tiles hold different rows, every K and V tile serves both.
//   narrow up to 128 rows (few tokens: single ones, ends of prompts): both hold the same rows, X takes the K and V tiles of its
//          parity, and the output warps join the two results.  (The time of these units is the cache's bytes; what counts is that
//          the next copies are always on their way.)
// The other warps: four write the results (the softmax goes on to the next unit meanwhile), one issues the copies (K and V of a
// stage of the ring together, the query rows), one for each row tile its products.
//
// Masks: a unit ends with the tile of its block's last token; in the last tiles a row sees the tokens up to its own.  V rows
// behind the block's last token are cleared in shared memory, so that nothing in the pages behind it counts.
// A row's reference is its running maximum, moved only when a logit exceeds it by more than 2^8.  P is rounded to bf16, the operand
// type of V: a weight is off by 3.9e-3 of itself at most, a row of random weights by 1.6e-3 on average, as much as by the output's own
// rounding.  The row sum adds the rounded weights, so that the rounding cancels where it is common to a row (one heavy
// weight, many equal ones; a value that all positions share comes back exactly).  The sum of the weights before their rounding
// leaves up to 3.9e-3 of such a row and is 1.5 % faster with heads of 128 (16384 tokens 1727 us instead of 1755), 3 to 5 % with
// heads of 64.  A second term of the weights, as the forest attention has it for heads of 64, would be a second product of O and
// more instructions for the softmax, which bound heads of 64 here already.
//
// Work split: the tiles of all units form one sequence (sequence, KV head, block), cut into runs of equal cost, one per CTA; a unit
// that straddles a cut leaves partial results that k_chunk_merge joins.  Few short units are taken whole, one a CTA.  Every
// CTA finds its run with one scan over the sequences; there is no plan kernel.
//
// What bounds it: wide units shared memory's bandwidth (96 KB of operands of S, 32 KB of V and 32 KB of copies for 64 tokens of both row
// tiles, 1545 cycles, where the products alone take 1100) and, in calls of a millisecond, the power limit: 16384 tokens at once, 32 / 8
// heads of 128, 1.72 ms (1280 TFLOP/s), 2.00 ms (1100) in a loop of seconds, where the clock falls to 1.4 GHz.  Single tokens HBM:
// 64 behind 1024 to 4096 97 us, 6.0 TB/s.  The shortest calls a chain of latencies: 4 tokens behind 512, heads of 64, 9.0 to 9.5 us.
//
// Every mbarrier wait is bounded; on a time-out the kernel records DSBD_DEV_TIMEOUT, lets its copies and products land,
// frees its TMEM and returns.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "dsbd_tc.cuh"

using namespace dsbd;

namespace {

constexpr int kRows = 128;                           // rows of a row tile
constexpr int kTile = kBN;                           // tokens of a tile: a page
constexpr int kPartRows = 2 * kRows;                 // rows of a unit
constexpr int kThreads = 512;                        // two softmax warpgroups, the output's, one with producer and issuers
constexpr int kWarpOut = 8, kWarpTma = 12, kWarpMma = 13;      // kWarpMma + X issues the products of row tile X
constexpr uint32_t kTmemCols = 512, kColS = 0, kColO = 256;    // S: [X][2 buffers][kTile]
constexpr float kMoveRef = 8.f;
#ifdef DSBD_TEST_WAIT_TIMEOUT
constexpr uint32_t kWaitTries = 250;                 // test build: see dsbd_attention_tr.cu
#else
constexpr uint32_t kWaitTries = 500000;              // about two seconds: a try is suspended for 4 us
#endif

template <int D>
struct Shape {
    static constexpr int kHalves = D / 64;
    static constexpr uint32_t kQHalf = kRows * 128, kQ = kHalves * kQHalf;       // 64 columns of a row tile; a row tile
    static constexpr uint32_t kHalf = kTile * 128, kKv = kHalves * kHalf;        // 64 columns of a K or V tile; a tile
    static constexpr uint32_t kStage = 2 * kKv;                                  // K then V
    static constexpr int kStages = D == 128 ? 5 : 8;
    static constexpr uint32_t kSmem = 2 * kQ + kStages * kStage;
};

// Costs are counted in tokens that a block's rows see, kNarrowShare of them in narrow units: a wide tile takes 1545 cycles, a
// narrow one half as long where HBM does not hold it up (its row tiles share the tokens) and 1400 where all SMs read their
// caches at once.  A unit's beginning and end are worth kWideCost and kNarrowCost more.  Batches of chunks and single tokens are
// up to 12 % faster than with a share of 1 (12 chunks of 1 to 777 tokens behind 0 to 6000: 100.6 us -> 97.1), the rest as fast; 0.5 gains as much
// on those and loses 10 % on many short chunks.
constexpr int kWideCost = 192, kNarrowCost = 288;
constexpr double kNarrowShare = 0.75;
constexpr int kMinRun = 384;                         // smallest run

struct ChunkArgs {
    int B, Hq, Hkv, group, T, max_new;
    int tile_tokens, block_tokens;                   // tokens of a row tile (128 / group) and of a block (two)
    int box_tokens;                                  // of a query box
    int whole, max_blocks;                           // a unit a CTA, nothing is cut: (sequence, KV head, one of max_blocks blocks)
    double per_block;                                // 1 / block_tokens
    float scale_log2;
    int64_t max_len, n_pages;
    const int32_t *new_off, *page_table;
    const int64_t *prefix_off, *page_off;
    __nv_bfloat16 *out;
    int out32;                                       // out is 32-byte aligned
    int32_t *status;
    struct CutRec *recs;                             // [grid]
    // what parts of units leave, run i's in slot 2 i (a unit that an earlier run began) and 2 i + 1 (one that it began):
    float *part_ml, *part_o;                         // [2 * grid][kPartRows][2] reference and row sum, [..][D] O
};

// A place in the work: unit (b, g, q) and a tile of it.
struct Pos { int b, g, q, t; };
__device__ __forceinline__ bool before(const Pos &x, const Pos &y) {
    if (x.b != y.b) return x.b < y.b;
    if (x.g != y.g) return x.g < y.g;
    if (x.q != y.q) return x.q < y.q;
    return x.t < y.t;
}

// What a run left for the merge.  tail: a unit that it began and did not end, of `tokens` rows of the tensors from `first` on and KV head g;
// head: how it went on with one that an earlier run began (0 not at all, 1 not to its end, 2 to its end).
struct CutRec { int tail, head, first, tokens, g, pad[3]; };

struct Seq { int n, first; int64_t L; };
__device__ __forceinline__ Seq seq_of(const ChunkArgs &a, int b, bool tell) {
    Seq s;
    s.first = a.new_off[b];
    const int end = a.new_off[b + 1];
    s.L = a.prefix_off[b + 1] - a.prefix_off[b];
    s.n = end - s.first;
    if (s.first < 0 || end < s.first || end > a.T || s.n > a.max_new || s.L < 0 || s.L > a.max_len || s.L + s.n > a.max_len) {
        s.n = 0;
        if (tell) report(a.status, DSBD_DEV_BAD_CHUNK);
    }
    return s;
}
// ceil(n / block_tokens): half a token more keeps the product off the whole numbers, from which its error is far smaller.
__device__ __forceinline__ int blocks_of(const ChunkArgs &a, int n) {
    return n == 0 ? 0 : (int)(((double)(n - 1) + 0.5) * a.per_block) + 1;
}
// Cost of the first q < blocks_of(n) blocks of one head of a sequence, and of all (a last block of at most tile_tokens is narrow).
__device__ __forceinline__ double cost_before(const ChunkArgs &a, const Seq &s, int q) {
    return (double)q * ((double)(s.L + kWideCost) + (double)a.block_tokens * 0.5 * (double)(q + 1));
}
__device__ __forceinline__ bool narrow_block(const ChunkArgs &a, const Seq &s, int q) {
    return s.n - q * a.block_tokens <= a.tile_tokens;
}
__device__ __forceinline__ double head_cost(const ChunkArgs &a, const Seq &s) {
    const int last = blocks_of(a, s.n) - 1;
    if (last < 0) return 0.0;
    const double sees = (double)(s.L + s.n);
    return floor(cost_before(a, s, last) + (narrow_block(a, s, last) ? kNarrowCost + kNarrowShare * sees : kWideCost + sees));
}

struct Unit {
    int first, n;                                    // rows of the sequence
    int64_t L;
    int i0, tokens;                                  // the block's first token and number of tokens
    int64_t end;                                     // tokens that the block's last one sees
    int nt;
    bool wide;
    int step, ahead;                                 // tiles from one of a row tile to its next; tiles that S runs ahead of O (two of a row tile)
};
__device__ __forceinline__ Unit unit_of(const ChunkArgs &a, const Seq &s, int q) {
    Unit u;
    u.first = s.first; u.n = s.n; u.L = s.L;
    u.i0 = q * a.block_tokens;
    u.tokens = min(a.block_tokens, s.n - u.i0);
    u.end = s.L + u.i0 + u.tokens;
    u.nt = (int)((u.end + kTile - 1) / kTile);
    u.wide = u.tokens > a.tile_tokens;
    u.step = u.wide ? 1 : 2;
    u.ahead = 2 * u.step;
    return u;
}

// Walks a run: the parts of units from `at` to `end`.
struct Walk {
    Pos at, end;
    Seq s;
    int nq;
    __device__ __forceinline__ void start(const ChunkArgs &a, const Pos &p0, const Pos &p1, const Seq &s0) {
        at = p0; end = p1;
        if (before(at, end)) { s = s0; nq = blocks_of(a, s.n); }
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

struct Shared {
    unsigned long long full[2][8], empty[2][8], s_full[2][2], p_full[2][2], ml_full[2], o_full[2], o_free[2], q_full, q_empty, drain[2];
    uint32_t tmem_base;
    int abort;
    Pos start, end;
    Seq seq;                                         // of start.b, and its pages
    int64_t table0, n_table;
    float2 ml[2][kRows];                             // [X] reference and row sum of the rows
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

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
          "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
// Products and commits are issued by one lane that elect.sync names (the same one for the same warp): its operands are uniform
// for the compiler.  An MMA takes 36 cycles to issue so, 62 with one lane's predicate on a converged warp's instruction
// (M = 128, N = 16, K = 16; at N = 64 and 128 43 and 59 cycles, what it takes to run).
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void mma_ss_one(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void mma_ts_one(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void commit_one(void *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// 32 bytes a lane (32-byte aligned): a warp's rows lie far apart, so a store instruction costs a line per lane.
__device__ __forceinline__ void st_32b(void *p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

// Stage number `seq` of the ring: its slot, the barriers of its landing and of its release, their phase.  A slot has two pairs of
// barriers, for its fillings in turn: a warp that does not use every stage (narrow units) may wait for a filling while the
// one before it, the other row tile's, is still on its way (copies land in any order), or ask for a release when the next
// filling is done with already, and the parity of one barrier could not tell neighbours apart.  Fillings two apart it need not:
// stage n - 2 STAGES had been released when n - STAGES was filled, and who waits for n has seen one later than that (a stage
// of its own or the part's query rows); and nobody gets past stage n + STAGES while a row tile still works on n.
template <int STAGES>
struct Stage {
    uint32_t slot, filling;
    __device__ __forceinline__ explicit Stage(uint32_t seq) : slot(seq % STAGES), filling(seq / STAGES) {}
    __device__ __forceinline__ void *full(Shared *sh) const { return &sh->full[filling & 1][slot]; }
    __device__ __forceinline__ void *empty(Shared *sh) const { return &sh->empty[filling & 1][slot]; }
    __device__ __forceinline__ uint32_t parity() const { return (filling >> 1) & 1; }
};

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
// NaN if any of the three is.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// 2^z for z <= 120 on the FMA and integer pipes, which are idle while ex2 (a quarter of a warp's lanes a cycle) sets the pace:
// z = n + f with n the nearest integer (what 1.5 * 2^23 leaves in the low bits), 2^f by a cubic fitted to the smallest relative
// error on [-1/2, 1/2] with 1 at f = 0 (1.0e-4; the weights are rounded to bf16, 3.9e-3), n into the exponent.
// From -127 down, -infinity included, the result is 0; for a NaN it is 0 too (the integer addition would make a number of it
// in any case), so a row's NaN is noticed by its maximum.
__device__ __forceinline__ F2 exp2_poly(F2 z) {
    const F2 big = {12582912.f, 12582912.f};
    z.x = fmaxf(z.x, -127.f);
    z.y = fmaxf(z.y, -127.f);
    const F2 r = add2(z, big);
    const F2 n = add2(r, F2{-12582912.f, -12582912.f});
    const F2 f = fma2(n, F2{-1.f, -1.f}, z);
    F2 p = fma2(f, F2{0.05500893294811249f, 0.05500893294811249f}, F2{0.2422109693288803f, 0.2422109693288803f});
    p = fma2(p, f, F2{0.6932829022407532f, 0.6932829022407532f});
    p = fma2(p, f, F2{1.f, 1.f});
    return F2{__uint_as_float(__float_as_uint(p.x) + (__float_as_uint(r.x) << 23)),
              __uint_as_float(__float_as_uint(p.y) + (__float_as_uint(r.y) << 23))};
}
constexpr int kPolyOf8 = 2;                          // of eight pairs of weights, those taken by exp2_poly

// The CTA's run, by one warp.  Returns through sh.start, sh.end, sh.seq and the pages' range; the sequences' facts are checked here, once
// a launch.  This stands before everything else of a call, and most of its time is that of fetching its instructions: one round
// of loads, doubles in place of 64-bit integers, quotients by floats that steps put right (8500 cycles without that).
__device__ void find_run(const ChunkArgs &a, Shared &sh) {
    const int lane = threadIdx.x & 31;
    if (a.whole) {
        const int c = (int)blockIdx.x, pair = c / a.max_blocks;
        Pos p;
        p.b = pair / a.Hkv; p.g = pair - p.b * a.Hkv; p.q = c - pair * a.max_blocks; p.t = 0;
        const int64_t table0 = a.page_off[p.b], table1 = a.page_off[p.b + 1];
        const Seq s = seq_of(a, p.b, p.g == 0 && p.q == 0 && lane == 0);
        if (lane == 0) {
            sh.start = sh.end = p;
            if (p.q < blocks_of(a, s.n)) ++sh.end.q;
            sh.seq = s;
            sh.table0 = table0;
            sh.n_table = table1 - table0;
        }
        return;
    }
    const int per = (a.B + 31) / 32, b0 = min(lane * per, a.B), b1 = min(b0 + per, a.B);
    // (a lane's first sequence stays in registers: the only one up to 32)
    Seq s0 = {};
    int64_t table0 = 0, table1 = 0;
    double hc0 = 0.0;
    if (b0 < b1) {
        table0 = a.page_off[b0];
        table1 = a.page_off[b0 + 1];
        s0 = seq_of(a, b0, blockIdx.x == 0);
        hc0 = head_cost(a, s0);
    }
    double sum = hc0 * a.Hkv;
#pragma unroll 1
    for (int b = b0 + 1; b < b1; ++b) sum += head_cost(a, seq_of(a, b, blockIdx.x == 0)) * a.Hkv;
    const double hi = warp_scan(sum, lane), lo = hi - sum, total = __shfl_sync(kFull, hi, 31);
    // the cuts: equal runs, not too small.  (A CTA and its neighbour work the cut between them out alike.)
    const int runs = max(1, (int)fmin((double)gridDim.x, floor(total * (1.0 / kMinRun))));
    const double share = total * (double)__frcp_rn((float)runs);         // (the last cut is the total itself)
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
        const int c = (int)blockIdx.x + k;
        const double cut = c >= runs ? total : floor((double)c * share);
        if (lane == 0) {
            const Pos over = {a.B, 0, 0, 0};
            (k == 0 ? sh.start : sh.end) = over;
        }
        __syncwarp();
        if (cut < lo || cut >= hi) continue;
        double in = cut - lo, hc = hc0;
        Seq s = s0;
        int b = b0;
#pragma unroll 1
        while (in >= hc * a.Hkv) {                   // (cut < hi: it lies in one of the sequences)
            in -= hc * a.Hkv;
            s = seq_of(a, ++b, false);
            hc = head_cost(a, s);
        }
        Pos p;
        p.b = b;
        p.g = max((int)__fdividef((float)in, (float)hc) - 1, 0);
        while ((double)(p.g + 1) * hc <= in) ++p.g;
        in -= (double)p.g * hc;
        // largest q with cost_before(q) <= in: the root of a quadratic
        const int nq = blocks_of(a, s.n);
        const float per_block = (float)a.per_block, h = (float)(s.L + kWideCost) * per_block + 0.5f;
        float root;
        asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(h * h + 2.f * (float)in * per_block));
        p.q = max(min((int)(root - h), nq) - 2, 0);
        while (p.q + 1 < nq && cost_before(a, s, p.q + 1) <= in) ++p.q;
        // (what a unit costs beside its tokens lies before them)
        in -= cost_before(a, s, p.q);
        p.t = narrow_block(a, s, p.q) ? max((int)((in - kNarrowCost) * (1.0 / (kNarrowShare * kTile))), 0)
                                      : max((int)((in - kWideCost) * (1.0 / kTile)), 0);
        if (k == 0) {
            sh.start = p;
            sh.seq = s;
            if (b != b0) { table0 = a.page_off[b]; table1 = a.page_off[b + 1]; }
            sh.table0 = table0;
            sh.n_table = table1 - table0;
        } else {
            sh.end = p;
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
k_chunk_attn(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
             const __grid_constant__ CUtensorMap map_q, ChunkArgs a) {
    using S = Shape<D>;
    using Stg = Stage<S::kStages>;
    extern __shared__ __align__(1024) unsigned char smem[];
    unsigned char *q_s = smem, *ring = smem + 2 * S::kQ;
    __shared__ Shared sh;
    const int warp = __shfl_sync(kFull, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    if ((smem_u32(smem) & 1023u) != 0u) {                    // the swizzled operands need 1024-byte alignment
        if (threadIdx.x == 0) report(a.status, DSBD_DEV_BAD_CHUNK);
        if (threadIdx.x == 0 && a.recs) a.recs[blockIdx.x] = CutRec{};
        return;
    }
    static_assert(sizeof(Shared) <= 3072 && 3072 + S::kSmem <= 227 * 1024, "both in the shared memory of a block");

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) { mbar_init(&sh.full[0][s], 1); mbar_init(&sh.full[1][s], 1); mbar_init(&sh.empty[0][s], 2); mbar_init(&sh.empty[1][s], 2); }
        for (int x = 0; x < 2; ++x) {
            for (int k = 0; k < 2; ++k) { mbar_init(&sh.s_full[x][k], 1); mbar_init(&sh.p_full[x][k], 4); }
            mbar_init(&sh.ml_full[x], 4); mbar_init(&sh.o_full[x], 1); mbar_init(&sh.o_free[x], 4);
            mbar_init(&sh.drain[x], 1);
        }
        mbar_init(&sh.q_full, 1);
        mbar_init(&sh.q_empty, 2);
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kWarpMma) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)),
                     "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (warp == 0) find_run(a, sh);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(&sh.tmem_base);

    if (warp == kThreads / 32 - 1 && lane == 0 && a.recs) {              // (a warp without work)
        CutRec r = {};
        const Pos p0 = sh.start, p1 = sh.end;
        const bool same = p0.b == p1.b && p0.g == p1.g && p0.q == p1.q;
        r.tail = p1.t > 0 && (!same || p0.t == 0);
        r.head = p0.t == 0 ? 0 : !same ? 2 : p1.t > p0.t ? 1 : 0;
        if (r.tail) {
            const Unit u = unit_of(a, seq_of(a, p1.b, false), p1.q);
            r.first = u.first + u.i0; r.tokens = u.tokens; r.g = p1.g;
        }
        a.recs[blockIdx.x] = r;
    }

    Walk w;
    w.start(a, sh.start, sh.end, sh.seq);
    if (warp == kWarpTma) {
        // ------------------------------------------------------------ copies
        // A part of nt tiles takes nt + ahead stages: stage j has V tile j - ahead and K tile j, where there are such.
        uint32_t seq = 0, part = 0;
        bool ok = true;
        int table_b = sh.start.b;
        int64_t table0 = sh.table0, n_table = sh.n_table;
        for (; ok && w.more(); w.next(a, a.Hkv)) {
            const Unit u = unit_of(a, w.s, w.at.q);
            const int t0 = w.at.t, nt = w.last_tile(u) - t0, g = w.at.g;
            if (nt <= 0) continue;
            const bool on = lane == 0;
            // K and V of a sequence with one block of rows pass once
            uint64_t policy;
            if (w.nq == 1) asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
            else asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
            // page ids: 32 in a warp's registers, those of the 32 pages before for the V tiles, which come later
            if (w.at.b != table_b) {
                table_b = w.at.b;
                table0 = a.page_off[table_b];
                n_table = a.page_off[table_b + 1] - table0;
            }
            auto fetch = [&](int from) -> int {
                const int p = from + lane;
                int id = -1;
                if (p < t0 + nt) {
                    if (p < n_table) {
                        id = a.page_table[table0 + p];
                        if (id < 0 || id >= a.n_pages) { report(a.status, DSBD_DEV_BAD_CHUNK); id = -1; }
                    } else {
                        report(a.status, DSBD_DEV_CAPACITY);
                    }
                }
                return id;
            };
            int ids = fetch(t0), before_ids = ids, at = 0;
            auto row_of = [&](int tile) -> int {                 // of the pools' maps (past their ends: zeros)
                const int id = __shfl_sync(kFull, tile >= at ? ids : before_ids, tile & 31);
                return id < 0 ? INT32_MAX - 2 * kBN : (id * a.Hkv + g) * kBN;
            };
            for (int j = 0; j < nt + u.ahead && ok; ++j) {
                if (j == 2) {
                    // (the first K tile of either row tile does not wait for the query rows of the part before to be done with)
                    if (part > 0) ok = warp_wait(&sh.q_empty, (part - 1) & 1, &sh);
                    if (!ok) break;
                    ++part;
                    const int tiles = u.wide ? 2 : 1;
                    mbar_expect_tx_if(on, &sh.q_full, (uint32_t)(tiles * a.box_tokens * a.group * D * 2));
                    for (int x = 0; x < tiles; ++x)
#pragma unroll
                        for (int h = 0; h < S::kHalves; ++h)
                            tma_load_3d(on, smem_u32(q_s + x * S::kQ + h * S::kQHalf), &map_q, h * 64, g * a.group,
                                        u.first + u.i0 + x * a.tile_tokens, &sh.q_full);
                }
                if (j == at + 32) { before_ids = ids; at = j; ids = fetch(t0 + j); }
                const bool has_k = j < nt, has_v = j >= u.ahead;
                const Stg to(seq);
                if (to.filling > 0) {
                    const Stg from(seq - S::kStages);
                    ok = warp_wait(from.empty(&sh), from.parity(), &sh);
                    if (!ok) break;
                }
                const int yk = row_of(j), yv = row_of(max(j - u.ahead, 0));
                mbar_expect_tx_if(on, to.full(&sh), (uint32_t)(has_k + has_v) * S::kKv);
#ifdef DSBD_TEST_WAIT_TIMEOUT
                const bool there = !(seq == 1 && blockIdx.x == 0);       // the bytes this barrier expects never come
#else
                const bool there = true;
#endif
                const uint32_t dst = smem_u32(ring + to.slot * S::kStage);
#pragma unroll
                for (int h = 0; h < S::kHalves; ++h) {
                    tma_load_2d_hint(on && there && has_v, dst + S::kKv + h * S::kHalf, &map_v, h * 64, yv, to.full(&sh), policy);
                    tma_load_2d_hint(on && there && has_k, dst + h * S::kHalf, &map_k, h * 64, yk, to.full(&sh), policy);
                }
                ++seq;
            }
        }
        // the copies land before the CTA goes away, also where another warp gave up
        for (uint32_t k = 0; k < (uint32_t)S::kStages && k < seq; ++k) {
            const Stg t(seq - 1 - k);
            for (uint32_t i = 0; i < kWaitTries && !mbar_try(t.full(&sh), t.parity()); ++i) {}
        }
        if (part > 0)
            for (uint32_t i = 0; i < kWaitTries && !mbar_try(&sh.q_full, (part - 1) & 1); ++i) {}
    } else if (warp == kWarpMma || warp == kWarpMma + 1) {
        // ------------------------------------------------------------ products
        const int x = warp - kWarpMma;
        constexpr uint32_t idesc_s = instr_desc(kRows, kTile, 0, 0);
        constexpr uint32_t idesc_o = instr_desc(kRows, D, 0, 1);
        const uint32_t s_col = tmem + kColS + x * 2 * kTile, o_col = tmem + kColO + x * D;
        uint32_t base = 0, part = 0, ns = 0, np = 0;             // stages before the part; S products and P's so far
        bool ok = true;
        for (; ok && w.more(); w.next(a, a.Hkv)) {
            const Unit u = unit_of(a, w.s, w.at.q);
            const int nt = w.last_tile(u) - w.at.t;
            if (nt <= 0) continue;
            // wide: this row tile takes every K and V tile, narrow: those of its parity
            const int step = u.step;
            ok = warp_wait(&sh.q_full, part & 1, &sh);
            const uint64_t qd = desc_k_major(smem_u32(q_s + (u.wide ? x : 0) * S::kQ));
            // (the elected lane's)
            auto product_s = [&](const Stg &t) {
                const uint64_t kd = desc_k_major(smem_u32(ring + t.slot * S::kStage));
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    mma_ss_one(s_col + (ns & 1) * kTile, qd + (uint64_t)((ks / 4) * (S::kQHalf >> 4) + (ks % 4) * 2),
                               kd + (uint64_t)((ks / 4) * (S::kHalf >> 4) + (ks % 4) * 2), idesc_s, ks > 0);
                commit_one(&sh.s_full[x][ns & 1]);
            };
            // a stage is free when both warps have told so: in narrow units the one that uses it tells for both
            auto release = [&](const Stg &t) {
                commit_one(t.empty(&sh));
                if (!u.wide) commit_one(t.empty(&sh));
            };
            int left = u.wide ? nt : (nt - x + 1) / 2;                   // S products to come
            const bool none = left == 0;
            // the stages of the first K tiles
            for (int j = u.wide ? 0 : x; j < u.ahead && ok; j += step) {
                const Stg t(base + j);
                ok = warp_wait(t.full(&sh), t.parity(), &sh);
                if (!ok) break;
                tc_fence_after();
                if (j < nt) --left;
                if (elect_one()) {
                    if (j < nt) {
                        product_s(t);
                        if (left == 0) commit_one(&sh.q_empty);
                        release(t);
                    } else {                                             // an empty stage
                        mbar_arrive(t.empty(&sh));
                        if (!u.wide) mbar_arrive(t.empty(&sh));
                    }
                }
                __syncwarp();
                if (j < nt) ++ns;
            }
            // (the accumulators of the part before have been read; every part waits, so that no phase is missed)
            if (ok && part > 0) ok = warp_wait(&sh.o_free[x], (part - 1) & 1, &sh);
            if (ok && none) {                                            // no tile of this parity
                if (elect_one()) { mbar_arrive(&sh.q_empty); mbar_arrive(&sh.o_full[x]); }
                __syncwarp();
            }
            for (int i = u.wide ? 0 : x; i < nt && ok; i += step) {
                const Stg t(base + u.ahead + i);
                ok = warp_wait(t.full(&sh), t.parity(), &sh) && warp_wait(&sh.p_full[x][np & 1], (np >> 1) & 1, &sh);
                if (!ok) break;
                tc_fence_after();
                const bool more = i + u.ahead < nt;
                left -= more;
                if (elect_one()) {
                    const uint64_t vd = desc_mn_major(smem_u32(ring + t.slot * S::kStage) + S::kKv, S::kHalf);
#pragma unroll
                    for (int ks = 0; ks < kTile / 16; ++ks)
                        mma_ts_one(o_col, s_col + (np & 1) * kTile + ks * 8, vd + (uint64_t)(ks * ((16 * 128) >> 4)), idesc_o,
                                   (i >= step || ks > 0) ? 1u : 0u);
                    if (more) {
                        product_s(t);
                        if (left == 0) commit_one(&sh.q_empty);
                    }
                    release(t);
                    if (i + step >= nt) commit_one(&sh.o_full[x]);
                }
                __syncwarp();
                ++np;
                ns += more;
            }
            base += nt + u.ahead;
            ++part;
        }
        // the block's shared memory outlives every arrival that the products have yet to make
        if (elect_one()) commit_one(&sh.drain[x]);
        __syncwarp();
        uint32_t i = 0;
        while (!__all_sync(kFull, mbar_try(&sh.drain[x], 0)) && i < kWaitTries) ++i;
    } else if (warp < kWarpOut) {
        // ------------------------------------------------------------ softmax
        const int x = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_base = tmem + lanes + kColS + x * 2 * kTile, o_addr = tmem + lanes + kColO + x * D;
        const int token = row / a.group;
        uint32_t base = 0, ns = 0, part = 0;
        bool ok = true;
        for (; ok && w.more(); w.next(a, a.Hkv)) {
            const Unit u = unit_of(a, w.s, w.at.q);
            const int t0 = w.at.t, nt = w.last_tile(u) - t0;
            if (nt <= 0) continue;
            const int i0 = u.i0 + (u.wide ? x * a.tile_tokens : 0);          // the row tile's first token
            const int left = min(a.tile_tokens, u.n - i0);                   // its tokens
            const bool work = (warp & 3) * 32 < left * a.group;              // some row of the warp
            // in tokens of the part: what this row sees, what every row of the tile sees, the block's end
            const int all_see = (int)(u.L - (int64_t)t0 * kTile) + i0 + 1, sees = all_see + token;
            const int end = (int)(u.end - (int64_t)t0 * kTile);
            const int step = u.step;
            float m_ref = -INFINITY, l = 0.f;
            for (int i = u.wide ? 0 : x; i < nt; i += step, ++ns) {
                const uint32_t s_addr = s_base + (ns & 1) * kTile;
                ok = warp_wait(&sh.s_full[x][ns & 1], (ns >> 1) & 1, &sh);
                if (!ok) break;
                tc_fence_after();
                // What lies behind the block's last token has weight zero: its values become zeros.  (In wide units by either group, before
                // its own product may run: which of the two comes first is open.)
                if ((i + 1) * kTile > end) {
                    const Stg t(base + u.ahead + i);
                    ok = warp_wait(t.full(&sh), t.parity(), &sh);
                    if (!ok) break;
                    if (row < kTile && row >= end - i * kTile) {
#pragma unroll
                        for (int h = 0; h < S::kHalves; ++h) {
                            uint4 *line = reinterpret_cast<uint4 *>(ring + t.slot * S::kStage + S::kKv + h * S::kHalf + row * 128);
#pragma unroll
                            for (int e = 0; e < 8; ++e) line[e] = make_uint4(0, 0, 0, 0);
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                if (work) {
                    uint32_t sv[2][32];
#pragma unroll
                    for (int c = 0; c < 2; ++c) tmem_ld32(s_addr + c * 32, sv[c]);
                    tmem_wait_ld();
                    if ((i + 1) * kTile > all_see) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const int lim = min(max(sees - i * kTile - c * 32, 0), 32);
                            const uint32_t vis = lim == 32 ? ~0u : (1u << lim) - 1;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!((vis >> e) & 1u)) sv[c][e] = 0xff800000u;      // -inf: weight 0
                        }
                    }
                    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < kTile; c += 2)
                        m4[(c >> 1) & 3] = max3(m4[(c >> 1) & 3], __uint_as_float(sv[c >> 5][c & 31]), __uint_as_float(sv[c >> 5][(c & 31) + 1]));
                    const float mx = max3(max3(m4[0], m4[1], m4[2]), m4[3], m4[3]) * a.scale_log2;      // scale > 0
                    const bool need = mx > m_ref + kMoveRef;         // (not for a NaN: the reference stays as it is)
                    if (__any_sync(kFull, need)) {
                        const float m_new = need ? mx : m_ref;
                        const float f = m_ref == -INFINITY ? 0.f : exp2f(m_ref - m_new);
                        l *= f;
                        if (i >= step) {
                            // the O product of the tile before has landed when that one's stage is free
                            const Stg t(base + u.ahead + i - step);
                            ok = warp_wait(t.empty(&sh), t.parity(), &sh);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {
                                uint32_t ov[16];
                                tmem_ld16(o_addr + c, ov);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 16; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * f);
                                tmem_st16(o_addr + c, ov);
                            }
                        }
                        m_ref = m_new;
                    }
                    const float neg = m_ref == -INFINITY ? 0.f : -m_ref;
                    F2 l2[2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t pv[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const F2 z = fma2(F2{__uint_as_float(sv[c][2 * e]), __uint_as_float(sv[c][2 * e + 1])},
                                              F2{a.scale_log2, a.scale_log2}, F2{neg, neg});
                            const F2 w2 = e % 8 < kPolyOf8 ? exp2_poly(z) : F2{ex2_ftz(z.x), ex2_ftz(z.y)};
                            pv[e] = pack_bf16(w2.x, w2.y);
                            l2[e & 1] = add2(l2[e & 1], F2{bf16_lo(pv[e]), bf16_hi(pv[e])});
                        }
                        tmem_st16(s_addr + c * 16, pv);
                    }
                    l += (l2[0].x + l2[0].y) + (l2[1].x + l2[1].y);
                    if (mx != mx) l = mx;                            // a logit that the row sees is NaN: so is its result, through every join
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.p_full[x][ns & 1]);
            }
            if (!ok) break;
            base += nt + u.ahead;
            // the row's reference and sum for the output warps, which have read those of the part before
            if (part > 0) ok = warp_wait(&sh.o_free[x], (part - 1) & 1, &sh);
            if (!ok) break;
            ++part;
            sh.ml[x][row] = make_float2(m_ref, l);
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.ml_full[x]);
        }
    } else if (warp < kWarpTma) {
        // ------------------------------------------------------------ output
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, o_addr = tmem + lanes + kColO;
        const int token = row / a.group, head = row - token * a.group;
        uint32_t part = 0;
        bool ok = true;
        for (; ok && w.more(); w.next(a, a.Hkv)) {
            const Unit u = unit_of(a, w.s, w.at.q);
            const int t0 = w.at.t, nt = w.last_tile(u) - t0;
            if (nt <= 0) continue;
            const bool is_whole = t0 == 0 && nt == u.nt;
#pragma unroll 1
            for (int x = 0; x < (u.wide ? 2 : 1) && ok; ++x) {
                const int i0 = u.i0 + x * a.tile_tokens;
                const bool active = token < min(a.tile_tokens, u.n - i0);
                const bool second = !u.wide && nt > 1;
                ok = warp_wait(&sh.ml_full[x], part & 1, &sh) && warp_wait(&sh.o_full[x], part & 1, &sh);
                if (ok && !u.wide) ok = warp_wait(&sh.ml_full[1], part & 1, &sh) && warp_wait(&sh.o_full[1], part & 1, &sh);
                if (!ok) break;
                tc_fence_after();
                float2 ml = sh.ml[x][row];
                float fo = 1.f, fb = 0.f;                    // factors of this tile's O and of the narrow unit's other one
                if (!u.wide) {
                    const float2 mb = sh.ml[1][row];
                    const float m = fmaxf(ml.x, mb.x);
                    fo = ml.x == -INFINITY ? 0.f : exp2f(ml.x - m);
                    fb = mb.x == -INFINITY ? 0.f : exp2f(mb.x - m);
                    ml = make_float2(m, ml.y * fo + mb.y * fb);
                }
                const int64_t at = (2 * (int64_t)blockIdx.x + (t0 == 0 ? 1 : 0)) * kPartRows + x * a.tile_tokens * a.group + row;
                float *part_o = a.part_o + at * D;
                __nv_bfloat16 *dst = a.out + ((int64_t)(u.first + i0 + token) * a.Hq + w.at.g * a.group + head) * D;
                if (is_whole) {
                    const float inv = 1.f / ml.y;
                    fo *= inv; fb *= inv;
                } else if (active) {
                    *reinterpret_cast<float2 *>(a.part_ml + at * 2) = ml;
                }
                // columns c .. c + C - 1 of the row: a TMEM load's latency shows once for all of them
                auto write = [&](auto cols, auto both, int c) {
                    constexpr int C = decltype(cols)::value;
                    uint32_t ov[C / 16][16], ow[C / 16][16];
#pragma unroll
                    for (int k = 0; k < C / 16; ++k) {
                        tmem_ld16(o_addr + x * D + c + 16 * k, ov[k]);
                        if (decltype(both)::value) tmem_ld16(o_addr + D + c + 16 * k, ow[k]);
                    }
                    tmem_wait_ld();
                    if (c + C == D) {                        // all read
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) {
                            mbar_arrive(&sh.o_free[x]);
                            if (!u.wide) mbar_arrive(&sh.o_free[1]);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < C / 16; ++k) {
                        float o[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            o[e] = __uint_as_float(ov[k][e]) * fo;
                            if (decltype(both)::value) o[e] = fmaf(__uint_as_float(ow[k][e]), fb, o[e]);
                        }
                        const int at = c + 16 * k;
                        if (active && is_whole) {
                            uint32_t w8[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) w8[e] = pack_bf16(o[2 * e], o[2 * e + 1]);
                            if (a.out32) {
                                st_32b(dst + at, w8);
                            } else {
                                *reinterpret_cast<uint4 *>(dst + at) = make_uint4(w8[0], w8[1], w8[2], w8[3]);
                                *reinterpret_cast<uint4 *>(dst + at + 8) = make_uint4(w8[4], w8[5], w8[6], w8[7]);
                            }
                        } else if (active) {
#pragma unroll
                            for (int e = 0; e < 16; e += 8) {
                                uint32_t w8[8];
#pragma unroll
                                for (int i = 0; i < 8; ++i) w8[i] = __float_as_uint(o[e + i]);
                                st_32b(part_o + at + e, w8);
                            }
                        }
                    }
                    __syncwarp();
                };
                if (second) {
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) write(std::integral_constant<int, 32>{}, std::true_type{}, c);
                } else {
#pragma unroll 1
                    for (int c = 0; c < D; c += 64) write(std::integral_constant<int, 64>{}, std::false_type{}, c);
                }
            }
            ++part;
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

// Joins the parts of cut units: block (i, y) takes rows of the unit that run i began and did not end, a warp to a row;
// out = sum_p O_p 2^(m_p - m) / sum_p l_p 2^(m_p - m), the parts in the order of their runs.  A call's time here is the chain of
// dependent loads, so the runs' records and the parts' references are read by a lane each, and the rows of O four at a time.
constexpr int kMergeThreads = 256, kMergeRows = kMergeThreads / 32;
template <int D>
__global__ void __launch_bounds__(kMergeThreads)
k_chunk_merge(ChunkArgs a, int runs) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int i0 = blockIdx.x, lane = threadIdx.x & 31;
    const int row = blockIdx.y * kMergeRows + (threadIdx.x >> 5);
    const CutRec rec = a.recs[i0];
    int next = i0 + 1 + lane < runs ? a.recs[i0 + 1 + lane].head : 2;
    if (!rec.tail) return;
    if (row >= rec.tokens * a.group) return;
    // the runs behind i0 that hold parts of the unit: those up to the first that ends it
    int parts = 1;
    for (;;) {
        const unsigned ends = __ballot_sync(kFull, next != 1);
        if (ends) {
            const int k = __ffs(ends) - 1;
            parts += k + (__shfl_sync(kFull, next, k) == 2 && i0 + parts + k < runs ? 1 : 0);
            break;
        }
        parts += 32;
        next = i0 + parts + lane < runs ? a.recs[i0 + parts + lane].head : 2;
    }
    constexpr int kPer = D / 32;
    float m = -INFINITY, l = 0.f, o[kPer] = {};
    for (int p0 = 0; p0 < parts; p0 += 32) {
        const int n = min(32, parts - p0);
        auto slot = [&](int p) { return 2 * (int64_t)(i0 + p0 + p) + (p0 + p == 0 ? 1 : 0); };
        float2 ml = {-INFINITY, 0.f};
        if (lane < n) ml = *reinterpret_cast<const float2 *>(a.part_ml + (slot(lane) * kPartRows + row) * 2);
        const float m_new = fmaxf(m, warp_max(ml.x));
        const float old = m == -INFINITY ? 0.f : exp2f(m - m_new);
        const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - m_new);
        l = l * old + warp_sum(ml.y * f);
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] *= old;
        m = m_new;
        for (int p = 0; p < n; p += 4) {
            float v[4][kPer], w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                w[k] = __shfl_sync(kFull, f, min(p + k, 31));
                const float *src = a.part_o + (slot(min(p + k, n - 1)) * kPartRows + row) * D + lane * kPer;
                if constexpr (kPer == 4) {
                    const float4 t = *reinterpret_cast<const float4 *>(src);
                    v[k][0] = t.x; v[k][1] = t.y; v[k][2] = t.z; v[k][3] = t.w;
                } else {
                    const float2 t = *reinterpret_cast<const float2 *>(src);
                    v[k][0] = t.x; v[k][1] = t.y;
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (p + k < n && w[k] != 0.f) o[e] = fmaf(v[k][e], w[k], o[e]);
        }
    }
    const float inv = 1.f / l;
    const int token = row / a.group, head = row - token * a.group;
    uint32_t *dst = reinterpret_cast<uint32_t *>(
        a.out + ((int64_t)(rec.first + token) * a.Hq + rec.g * a.group + head) * D + lane * kPer);
#pragma unroll
    for (int e = 0; e < kPer; e += 2) dst[e / 2] = pack_bf16(o[e] * inv, o[e + 1] * inv);
}

// Launch shape shared by the workspace query and the launch.
struct Plan { int grid, whole, max_blocks, block_rows; };
// Longest units that are taken whole where there is a CTA for each: 16 sequences of 1000 tokens x 8 heads 16.7 us whole and 21.5 cut, 4 of 1400
// 15.9 and 14.4 (a cut costs the merge, which is 5 us of a short call).
constexpr int64_t kWholeTokens = 1200;

Plan make_plan(const dsbd_chunk_t *c, const dsbd_attn_desc_t *d) {
    Plan p = {};
    int dev = 0, sms = 148;
    if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    const int group = d->Hq / d->Hkv, block = 2 * (kRows / group);
    p.block_rows = (int)std::min<int64_t>(block, c->max_new) * group;
    p.max_blocks = (int)((std::min<int64_t>(c->max_new, c->total_new) + block - 1) / block);
    const int64_t units = (int64_t)c->B * d->Hkv * p.max_blocks;         // (or places for them)
    p.whole = units <= sms && c->max_len <= kWholeTokens;
    p.grid = p.whole ? (int)units : sms;
    return p;
}

int check(const dsbd_chunk_t *c, const dsbd_attn_desc_t *d) {
    if (!c || !d || c->B <= 0 || !c->new_off || !c->prefix_off || c->total_new < 0 || c->max_new < 0 || (c->total_new > 0 && c->max_new == 0) || c->max_len < 0)
        return DSBD_ERR_INVALID_ARG;
    if (d->Hq <= 0 || d->Hkv <= 0 || d->Hq % d->Hkv || !(d->scale > 0.f) || !std::isfinite(d->scale)) return DSBD_ERR_INVALID_ARG;
    if (d->dtype != DSBD_DTYPE_BF16 || (d->d != 64 && d->d != 128) || d->Hq / d->Hkv > kRows) return DSBD_ERR_UNSUPPORTED;
    if (c->max_len > (int64_t)1 << 30) return DSBD_ERR_UNSUPPORTED;
    return DSBD_OK;
}

// Workspace: records, references and sums, accumulators.
size_t recs_bytes(const Plan &p) { return align_up(sizeof(CutRec) * (size_t)p.grid, 256); }
size_t ml_bytes(const Plan &p) { return sizeof(float) * 2 * 2 * (size_t)p.grid * kPartRows; }
size_t workspace_of(const Plan &p, int d) {
    return p.whole ? 256 : recs_bytes(p) + ml_bytes(p) + sizeof(float) * 2 * (size_t)p.grid * kPartRows * d;
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
    cfg.gridDim = dim3((unsigned)p.grid, (unsigned)((p.block_rows + kMergeRows - 1) / kMergeRows));
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
    a.B = c->B; a.Hq = d->Hq; a.Hkv = d->Hkv; a.group = d->Hq / d->Hkv; a.T = c->total_new; a.max_new = c->max_new;
    a.tile_tokens = kRows / a.group;
    a.block_tokens = 2 * a.tile_tokens;
    a.per_block = 1.0 / a.block_tokens;
    a.box_tokens = std::min(a.tile_tokens, c->total_new);
    a.whole = plan.whole;
    a.max_blocks = std::max(plan.max_blocks, 1);
    a.scale_log2 = d->scale * 1.4426950408889634f;
    a.max_len = c->max_len; a.n_pages = pages->n_pages;
    a.new_off = c->new_off; a.prefix_off = c->prefix_off; a.page_table = pages->page_table; a.page_off = pages->page_off;
    a.out = static_cast<__nv_bfloat16 *>(out);
    a.out32 = (reinterpret_cast<uintptr_t>(out) & 31) == 0;
    a.status = status;
    if (!plan.whole) {
        unsigned char *ws = static_cast<unsigned char *>(workspace);
        a.recs = reinterpret_cast<CutRec *>(ws);
        a.part_ml = reinterpret_cast<float *>(ws + recs_bytes(plan));
        a.part_o = reinterpret_cast<float *>(ws + recs_bytes(plan) + ml_bytes(plan));
    }
    CUtensorMap maps[3];
    const uint64_t D = (uint64_t)d->d;
    if (!make_map(&maps[0], k_pool, D, (uint64_t)rows, D * 2) || !make_map(&maps[1], v_pool, D, (uint64_t)rows, D * 2) ||
        !make_map_q(&maps[2], q, D, (uint64_t)d->Hq, (uint64_t)c->total_new, (uint32_t)a.group, (uint32_t)a.box_tokens))
        return DSBD_ERR_CUDA;
    return d->d == 64 ? launch<64>(plan, maps, a, stream) : launch<128>(plan, maps, a, stream);
}
