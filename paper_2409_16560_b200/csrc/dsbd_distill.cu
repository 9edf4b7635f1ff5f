// Distillation of rows of logits from a teacher's entries, loss and gradient in one pass.
//
// A row belongs to a cluster of 1 to 8 CTAs, each of which reads its share for the sums and again for the gradient: the last part from registers, the
// first from shared memory, the rest while it is still in the L2.
//
// The tokens that the teacher names are marked by bits.  The others' softmax has a reference of its own (their largest logit):
// beside a named token of nearly all the mass their sum would vanish in 32 bits, and with it the loss's last term.  Terms of the
// sums are in 32 bits (2^-22 each), a thread's terms are added in 32, everything behind that, the teacher's softmax and the loss
// are in 64 bits: p log p - p log q cancels when the student is near the teacher.
#include <algorithm>

#include "dsbd_rows.cuh"

namespace dsbd {
namespace rows {
namespace {

constexpr int NT = 256;

struct DistillArgs {
    const void *logits;
    int64_t stride;
    int V, K, ctas, per, held;                     // held: words of a share in shared memory, at most
    float temperature;
    double inverse;                                // 1 / temperature
    const float *value;
    const int32_t *index;
    const float *rest, *weight;
    float *loss;
    void *grad;
    int64_t grad_stride;
    int32_t *status;
};

struct Sums {
    double others, named;                          // relative to the logits below
    float top_others, top_named;
};

struct Shared {
    Told<Sums> told;
    float teacher[NT / 32];
    float2 most[NT / 32];
    double others[NT / 32], named[NT / 32], entries[NT / 32], scratch[NT / 32];
    uint32_t named_twice;
};

// f(token of the share, word's elements) into the gradient's row, in aligned words.
template <class T, class F>
__device__ __forceinline__ void put_share(T *row, const Share &s, F f) {
    constexpr int P = kPer<T>;
    T *to = row + s.first;
    const int mis = (int)((reinterpret_cast<uintptr_t>(to) & 15) / sizeof(T));
    const int words = s.count > 0 ? (mis + s.count + P - 1) / P : 0;
    for (int w = threadIdx.x; w < words; w += NT) {
        const int at = w * P - mis;
        float g[P];
        f(at, g);
        if (at >= 0 && at + P <= s.count) {
            *reinterpret_cast<float4 *>(to + at) = pack(g);
        } else {
#pragma unroll
            for (int e = 0; e < P; ++e)
                if (at + e >= 0 && at + e < s.count) to[at + e] = T(g[e]);
        }
    }
}

// MINE entries of a thread: k = threadIdx.x + i * NT.  RESIDENT CTAs of an SM.  GRAD: with the gradient (the losses alone leave the
// registers of its last batch free: one text for both 2 per cent slower with 4608 rows of 128256 fp32, 5 with 517 of 50257 bf16 without).
//
// One reading and one writing of the logits are what it has to do: 4608 rows of 128256 fp32 998 us, 4.7 TB/s in both directions together, of
// 723 at the copy rate (from one GPU to another up to 1029); 2048 rows in bf16 273 us of 161.  592 rows of 128256 read 1.11 times the logits from
// HBM in fp32 and 1.29 times in bf16 (shares of 128 KB under way: 444 and 592).  What holds it up is a CTA's chain (some 12000 cycles: the teacher, the first words, two
// exchanges, 64-bit sums), which the SM's other CTAs cover in part, and the second reading, from the L2 for what is not held in shared memory.  (Held:
// all of it leaves one CTA of an SM, less is slower in the L2; rows' loads begun a row ahead, 1 to 8 rows a cluster: no gain; 512 threads: slower.)
// Without a gradient one reading: 517 rows of 50257 bf16 18.1 us of 8, fp32 28 of 16; 1024 of 128256 fp32 107 of 80.
//
// 64-bit chains are kept short and off the others' way (a dependent step takes some 40 cycles, a logarithm more than a thousand): the teacher's
// exponentials run while the first words are on their way, the student's sums are joined by lanes side by side, and logarithms are
// for the loss alone, which one CTA works out behind its share of the gradient.
template <class T, int MINE, int RESIDENT, bool GRAD>
__global__ void __launch_bounds__(NT, RESIDENT) k_distill(DistillArgs a) {
    constexpr int P = kPer<T>, D = kDeep<T>;
    extern __shared__ float4 mem[];
    __shared__ Shared sh;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    begun_arrive(a.ctas);
    const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    const int row = blockIdx.x / a.ctas, rank = blockIdx.x - row * a.ctas;
    uint32_t *named = reinterpret_cast<uint32_t *>(mem + a.held);      // a bit for each element of the share's words
    const T *z_row = static_cast<const T *>(a.logits) + (int64_t)row * a.stride;
    T *g_row = GRAD ? static_cast<T *>(a.grad) + (int64_t)row * a.grad_stride : nullptr;
    const Share s = share<T>(z_row, a.V, rank, a.per);
    const float weight = a.weight ? a.weight[row] : 1.f;
    const float *value = a.value + (int64_t)row * a.K;
    const int32_t *index = a.index + (int64_t)row * a.K;
    const float rest = a.rest ? a.rest[row] : -CUDART_INF_F;
    float t[MINE], z[MINE];                        // the teacher's entry; the student's logit, where this CTA needs it
    int at[MINE];                                  // token; -1: no entry
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        const int k = threadIdx.x + i * NT;
        at[i] = k < a.K ? index[k] : -1;
        t[i] = k < a.K ? value[k] : -CUDART_INF_F;
    }
    auto no_gradient = [&] {
        if constexpr (GRAD) put_share<T>(g_row, s, [](int, float (&g)[P]) {
#pragma unroll
            for (int e = 0; e < P; ++e) g[e] = 0.f;
        });
    };
    if (weight == 0.f) {
        no_gradient();
        if (rank == 0 && threadIdx.x == 0) a.loss[row] = 0.f;
        begun_wait(a.ctas);
        return;
    }
    float4 raw[D];
    load_batch<T, NT>(raw, z_row, s, 0);
    // ---- the teacher's entries
    if (threadIdx.x == 0) sh.named_twice = 0;
    for (int w = threadIdx.x; w < (s.words + D * NT - 1) / (D * NT) * NT; w += NT) named[w] = 0;
    float mine = -CUDART_INF_F;
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        if (at[i] < -1 || at[i] >= a.V) {
            if (rank == 0) report(a.status, DSBD_DEV_BAD_TOKEN);
            at[i] = -1;
        }
        if (at[i] < 0) t[i] = -CUDART_INF_F;
        mine = fmaxf(mine, t[i]);
    }
    auto here = [&](int token) { return token >= s.first && token < s.first + s.count; };
#pragma unroll
    for (int i = 0; i < MINE; ++i) z[i] = here(at[i]) || (rank == 0 && at[i] >= 0) ? value_of(z_row[at[i]]) : -CUDART_INF_F;
    mine = warp_most(mine);
    if (lane == 0) sh.teacher[warp] = mine;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MINE; ++i)
        if (here(at[i])) {
            const int pos = s.mis + at[i] - s.first;
            const uint32_t bit = 1u << (pos & 31);
            if (atomicOr(&named[pos >> 5], bit) & bit) sh.named_twice = 1;
        }
    double top_t = (double)rest;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) mine = fmaxf(mine, sh.teacher[w]);
    top_t = fmax(top_t, (double)mine * a.inverse);
    __syncthreads();
    // the teacher's masses relative to its largest one
    double e[MINE];
#pragma unroll
    for (int i = 0; i < MINE; ++i) e[i] = t[i] != -CUDART_INF_F ? exp((double)t[i] * a.inverse - top_t) : 0.0;
    const double e_rest = rest != -CUDART_INF_F ? exp((double)rest - top_t) : 0.0;
    // an entry whose token an earlier one has already named: the first one stands for all of them
    bool stands[MINE];
    const bool twice = sh.named_twice != 0;
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        stands[i] = here(at[i]);
        if (twice)
            for (int k = 0; stands[i] && k < (int)threadIdx.x + i * NT; ++k) stands[i] = index[k] != at[i];
    }
    // ---- the student's sums
    const double scale = 1.4426950408889634 * a.inverse;
    const float scale_f = (float)scale;
    Rest others;
    for (int w0 = 0; w0 < s.words;) {
        // the warp's 1024 elements of the batch have 32 words of marks
        const bool some = __any_sync(kFull, named[w0 * P / 32 + threadIdx.x] != 0);
        float top = -CUDART_INF_F;
#pragma unroll
        for (int u = 0; u < D; ++u) {
            const int w = batch_word<D>(w0, u);
            if (w < a.held) mem[w] = raw[u];
            float x[P];
            unpack(raw[u], x);
            if (some) {
                const uint32_t marks = named[w * P >> 5] >> (w * P & 31) & ((1u << P) - 1);
                if (marks) {
#pragma unroll
                    for (int i = 0; i < P; ++i) x[i] = marks >> i & 1 ? -CUDART_INF_F : x[i];
                    raw[u] = pack(x);
                }
            }
#pragma unroll
            for (int i = 0; i < P; ++i) top = fmaxf(top, x[i]);
        }
        others.add_words<T>(raw, top, scale_f);
        if ((w0 += D * NT) < s.words) load_batch<T, NT>(raw, z_row, s, w0);
    }
    float2 most = {others.high, -CUDART_INF_F};
#pragma unroll
    for (int i = 0; i < MINE; ++i)
        if (stands[i]) most.y = fmaxf(most.y, z[i]);
    const bool entries = warp * 32 < a.K;          // the warp has some
    most = {warp_most(most.x), entries ? warp_most(most.y) : -CUDART_INF_F};
    if (lane == 0) sh.most[warp] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) most = {fmaxf(most.x, sh.most[w].x), fmaxf(most.y, sh.most[w].y)};
    const double sum_others = warp_total(others.high == most.x ? others.sum : others.sum * exp2_fast((others.high - most.x) * scale_f));
    double sum_named = 0.0, sum_entries = 0.0;
    if (entries) {
        // (in 64 bits: the loss takes these tokens' log q from their logits themselves, so an error of their sum would stay in it)
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            // (+inf: no softmax, so NaN, as x - most gives it where such a logit is not named)
            if (stands[i] && z[i] != -CUDART_INF_F) sum_named += z[i] < CUDART_INF_F ? rescale(z[i], most.y, scale) : (double)CUDART_NAN_F;
            sum_entries += e[i];
        }
        sum_named = warp_total(sum_named);
        sum_entries = warp_total(sum_entries);
    }
    if (lane == 0) {
        sh.others[warp] = sum_others;
        sh.named[warp] = sum_named;
        sh.entries[warp] = sum_entries;
    }
    __syncthreads();
    Sums own = {0.0, 0.0, most.x, most.y};
    double teacher = e_rest;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        own.others += sh.others[w];
        own.named += sh.named[w];
        teacher += sh.entries[w];
    }
    begun_wait(a.ctas);
    int turn = 0;
    const Sums *all = tell(own, sh.told, turn, a.ctas, rank);
    // the others' sum relative to their largest logit, base; of all relative to the row's
    float base = all[0].top_others, top = all[0].top_named;
#pragma unroll
    for (int c = 1; c < kMaxCtas; ++c)
        if (c < a.ctas) {
            base = fmaxf(base, all[c].top_others);
            top = fmaxf(top, all[c].top_named);
        }
    top = fmaxf(top, base);
    auto worth = [&](float from, float to) { return from == to ? 1.0 : (double)exp2_fast((from - to) * scale_f); };
    double rest_sum = 0.0;
#pragma unroll
    for (int c = 0; c < kMaxCtas; ++c)
        if (c < a.ctas) rest_sum += all[c].others * worth(all[c].top_others, base);
    // (in 64 bits, as the named tokens' below: the loss takes the others' log from their own sum)
    const double others_top = rest_sum * rescale(base, top, scale);
    // the named tokens' sum (at most K): a CTA's to a lane
    const double told_named = lane < a.ctas ? all[lane].named * rescale(all[lane].top_named, top, scale) : 0.0;
    const double whole = others_top + warp_total(told_named * 0x1p-10) * 0x1p10;
    if (whole == 0.0 || teacher == 0.0) {
        no_gradient();
        if (rank == 0 && threadIdx.x == 0) {
            a.loss[row] = 0.f;
            report(a.status, DSBD_DEV_EXHAUSTED);
        }
        return;
    }
    const double per_whole = inverse_of(whole), per_teacher = inverse_of(teacher);
    // ---- the gradient: the others', then the named tokens' over it
    if constexpr (GRAD) {
        const double q = others_top * per_whole;
        const float factor_f = rest_sum != 0.0 ? (float)((double)weight * a.temperature * (a.rest ? q - e_rest * per_teacher : q) * inverse_of(rest_sum))
                                                : whole == whole ? 0.f : CUDART_NAN_F;
        if (base == -CUDART_INF_F) base = 0.f;
        const float2 base2 = {-base, -base}, scale2 = {scale_f, scale_f}, factor2 = {factor_f, factor_f};
        auto slope = [&](float (&x)[P]) {
#pragma unroll
            for (int i = 0; i < P; i += 2) {
                const float2 y = mul2(add2({x[i], x[i + 1]}, base2), scale2), g = mul2({exp2_fast(y.x), exp2_fast(y.y)}, factor2);
                x[i] = g.x;
                x[i + 1] = g.y;
            }
        };
        if (((reinterpret_cast<uintptr_t>(g_row) ^ reinterpret_cast<uintptr_t>(z_row)) & 15) == 0) {
            // words of the gradient lie as the logits' do
            float4 *to = reinterpret_cast<float4 *>(g_row + s.first - s.mis);
            // backwards, from the batch that is still in registers on, so that what was read last is read again first (4608 rows of 128256 fp32: 1069
            // us, so 1022)
            const int last = s.words > 0 ? (s.words - 1) / (D * NT) * (D * NT) : -1;
            for (int w0 = last; w0 >= 0; w0 -= D * NT) {
                if (w0 == last) {
                    // (in raw)
                } else if (w0 + D * NT <= a.held) {
#pragma unroll
                    for (int u = 0; u < D; ++u) raw[u] = mem[batch_word<D>(w0, u)];
                } else {
                    load_batch<T, NT>(raw, z_row, s, w0);
                }
#pragma unroll
                for (int u = 0; u < D; ++u) {
                    const int w = batch_word<D>(w0, u), first = w * P - s.mis;
                    float x[P];
                    unpack(raw[u], x);
                    slope(x);
                    if (first >= 0 && first + P <= s.count) {
                        __stcs(to + w, pack(x));
                    } else {
#pragma unroll
                        for (int i = 0; i < P; ++i)
                            if (first + i >= 0 && first + i < s.count) g_row[s.first + first + i] = T(x[i]);
                    }
                }
            }
        } else {
            put_share<T>(g_row, s, [&](int first, float (&x)[P]) {
#pragma unroll
                for (int i = 0; i < P; ++i)
                    x[i] = first + i >= 0 && first + i < s.count ? value_of(z_row[s.first + first + i]) : -CUDART_INF_F;
                slope(x);
            });
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < MINE; ++i)
            if (stands[i]) {
                double p = e[i];
                if (twice)
                    for (int k = threadIdx.x + i * NT + 1; k < a.K; ++k)
                        if (index[k] == at[i]) p += exp((double)value[k] * a.inverse - top_t);
                // (in 64 bits: near its teacher a student's q - p is a small difference.  Its exponential kept from the sum above, in registers or in
                // shared memory, takes longer: 2048 rows of 128256 bf16 278 and 274 us, so 273, by exponentials in 32 bits 268)
                const double q = rescale(z[i], top, scale) * per_whole;
                g_row[at[i]] = T((float)((double)weight * a.temperature * (q - p * per_teacher)));
            }
    }
    // ---- the loss: sum p (log p - log q), log p = t / T - log of the teacher's sum, log q = z / T - log of the student's
    if (rank) return;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < MINE; ++i)
        if (e[i] != 0.0) sum += e[i] * (((double)t[i] - (double)z[i]) * a.inverse);
    if (entries) sum = warp_sum(sum);
    if (lane == 0) sh.scratch[warp] = sum;
    __syncthreads();
    if (warp) return;
    sum = 0.0;
    for (int w = 0; w < NT / 32; ++w) sum += sh.scratch[w];
    const double v = log(lane == 0 ? whole : lane == 1 ? teacher : rest_sum);
    const double log_t = __shfl_sync(kFull, v, 1) + top_t, log_q = __shfl_sync(kFull, v, 0) + (double)top * a.inverse;
    const double log_others = __shfl_sync(kFull, v, 2) + (double)base * a.inverse - log_q;
    sum += (teacher - e_rest) * (log_q - log_t);
    if (e_rest != 0.0) sum += e_rest * ((double)rest - log_t - log_others);
    if (lane == 0) a.loss[row] = (float)((double)a.temperature * a.temperature * (sum * per_teacher));
}

// CTAs of a row: shares of up to 128 KB (a CTA's fixed chain, some 12000 cycles, counts for less than with smaller ones; with larger
// ones the rows under way outgrow the L2, from which what is not held is read again: 2048 rows of 128256 bf16, two CTAs each 273 us, one
// 309), and more where the SMs would stand idle.
inline Plan plan_distill(const dsbd_rows_t *r, int resident) {
    const int size = r->dtype == DSBD_DTYPE_F32 ? 4 : 2;
    Plan p;
    p.ctas = 1;
    while (p.ctas < kMaxCtas && (share_of(r->V, p.ctas) * size > 128 * 1024 ||
           (r->rows * 2 * (int64_t)p.ctas <= 148 * resident && share_of(r->V, 2 * p.ctas) >= NT * 16)))
        p.ctas *= 2;
    p.per = share_of(r->V, p.ctas);
    p.words = 0;
    return p;
}

template <class T, int RESIDENT, bool GRAD>
int run_distill(const dsbd_rows_t *r, DistillArgs &a, dsbd_stream_t stream) {
    constexpr int kBatch = NT * kDeep<T>, kHeld = 48 * 1024;
    constexpr int kMost = kHeld + (kLongestShare + kBatch - 1) / kBatch * NT * 4;
    const Plan p = plan_distill(r, RESIDENT);
    a.ctas = p.ctas;
    a.per = p.per;
    // whole batches of 32 elements a thread, as many as leave room for RESIDENT CTAs in an SM's 228 KB, of which each takes 1 more (2048 rows of 128256 bf16,
    // an earlier form: three batches and three CTAs 306 us, two and four 280), but the last, which stays in registers; without a gradient nothing is read twice
    const int batches = (p.per / kPer<T> + 1 + kBatch - 1) / kBatch, marks = batches * NT * 4;
    const int room = 228 * 1024 / RESIDENT - 1024 - (int)sizeof(Shared) - marks;
    a.held = GRAD ? std::min(batches - 1, std::min(room, kHeld) / 16 / kBatch) * kBatch : 0;
    const size_t bytes = (size_t)a.held * 16 + (size_t)marks;
    return a.K <= NT ? launch<kMost, NT>(k_distill<T, 1, RESIDENT, GRAD>, r->rows, p, bytes, a, stream)
                     : launch<kMost, NT>(k_distill<T, DSBD_MAX_TOP / NT, RESIDENT, GRAD>, r->rows, p, bytes, a, stream);
}

}  // namespace
}  // namespace rows
}  // namespace dsbd

using namespace dsbd::rows;

extern "C" int dsbd_distill(const dsbd_rows_t *rows, const dsbd_distill_params_t *p, float *loss, void *grad, int64_t grad_stride,
                            int32_t *status, dsbd_stream_t stream) {
    int rc = check_rows(rows);
    if (rc) return rc;
    if (!p || p->K <= 0 || p->K > rows->V || !scales(p->temperature) || !status) return DSBD_ERR_INVALID_ARG;
    if (grad && rows->rows > 1 && grad_stride < rows->V) return DSBD_ERR_INVALID_ARG;
    const int size = rows->dtype == DSBD_DTYPE_F32 ? 4 : 2;
    if (p->K > DSBD_MAX_TOP || (reinterpret_cast<uintptr_t>(grad) & (size - 1))) return DSBD_ERR_UNSUPPORTED;
    if (rows->rows == 0) return DSBD_OK;
    if (!rows->logits || !p->value || !p->index || !loss) return DSBD_ERR_INVALID_ARG;
    DistillArgs a = {};
    a.logits = rows->logits; a.stride = rows->row_stride; a.V = rows->V; a.K = p->K;
    a.temperature = p->temperature;
    a.inverse = 1.0 / (double)p->temperature;
    a.value = p->value; a.index = p->index; a.rest = p->rest; a.weight = p->weight;
    a.loss = loss; a.grad = grad; a.grad_stride = grad_stride; a.status = status;
    // Four CTAs of an SM where their registers last (517 rows of 50257 bf16 without gradients 18.1 us, with three 23.9; 2048 of 128256 with gradients
    // 273 and 287); with gradients in fp32 three (20 rows of 32000 6.6 us, with four and what they spill 8.0; 4608 of 128256 996 and 1000).
    if (rows->dtype == DSBD_DTYPE_BF16)
        return grad ? run_distill<__nv_bfloat16, 4, true>(rows, a, stream) : run_distill<__nv_bfloat16, 4, false>(rows, a, stream);
    return grad ? run_distill<float, 3, true>(rows, a, stream) : run_distill<float, 4, false>(rows, a, stream);
}
