// Distillation of rows of logits from a teacher's entries, loss and gradient in one pass.
//
// A row belongs to a cluster of 1 to 8 CTAs, which brings it into shared memory once (its gradient is written from there), so the
// call moves what it cannot do without: each logit in, each gradient out.
//
// The tokens that the teacher names are marked by bits.  The others' softmax has a reference of its own (their largest logit):
// beside a named token of nearly all the mass their sum would vanish in 32 bits, and with it the loss's last term.  Terms of the
// sums are in 32 bits (2^-22 each), a thread's terms are added in 32, everything behind that, the teacher's softmax and the loss
// are in 64 bits: p log p - p log q cancels when the student is near the teacher.
#include "dsbd_rows.cuh"

namespace dsbd {
namespace rows {
namespace {

constexpr int kMine = DSBD_MAX_TOP / kThreads;     // entries of a thread: k = threadIdx.x + i * kThreads

struct DistillArgs {
    const void *logits;
    int64_t stride;
    int V, K, ctas, per, words;
    float temperature;
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
    double scratch[kWarps];
    float scratch_f[kWarps];
    uint32_t named_twice;
};

// f(token of the share, word's elements) into the gradient's row, in aligned words.
template <class T, class F>
__device__ __forceinline__ void put_share(T *row, const Share &s, F f) {
    constexpr int P = kPer<T>;
    T *to = row + s.first;
    const int mis = (int)((reinterpret_cast<uintptr_t>(to) & 15) / sizeof(T));
    const int words = s.count > 0 ? (mis + s.count + P - 1) / P : 0;
    for (int w = threadIdx.x; w < words; w += kThreads) {
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

template <class T>
__global__ void __launch_bounds__(kThreads) k_distill(DistillArgs a) {
    constexpr int P = kPer<T>;
    extern __shared__ float4 mem[];
    __shared__ Shared sh;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    begun_arrive(a.ctas);
    const int row = blockIdx.x / a.ctas, rank = blockIdx.x - row * a.ctas;
    const T *z_row = static_cast<const T *>(a.logits) + (int64_t)row * a.stride;
    T *g_row = a.grad ? static_cast<T *>(a.grad) + (int64_t)row * a.grad_stride : nullptr;
    const Share s = share<T>(z_row, a.V, rank, a.per);
    uint32_t *named = reinterpret_cast<uint32_t *>(mem + a.words);     // a bit for each position of the share's words
    const T *z_mem = reinterpret_cast<const T *>(mem);
    const float weight = a.weight ? a.weight[row] : 1.f;
    auto no_gradient = [&] {
        if (g_row) put_share<T>(g_row, s, [](int, float (&g)[P]) {
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
    // ---- the teacher's entries and the share
    const float *value = a.value + (int64_t)row * a.K;
    const int32_t *index = a.index + (int64_t)row * a.K;
    const float rest = a.rest ? a.rest[row] : -CUDART_INF_F;
    float t[kMine];
    int at[kMine];                                 // token; -1: no entry
    float z[kMine];                                // the student's logit, where this CTA needs it
    bool here[kMine];                              // its token is in the share
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int k = threadIdx.x + i * kThreads;
        at[i] = k < a.K ? index[k] : -1;
        t[i] = k < a.K ? value[k] : -CUDART_INF_F;
    }
    if (threadIdx.x == 0) sh.named_twice = 0;
    for (int w = threadIdx.x; w <= s.words * P / 32; w += kThreads) named[w] = 0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        if (at[i] < -1 || at[i] >= a.V) {
            if (rank == 0) report(a.status, DSBD_DEV_BAD_TOKEN);
            at[i] = -1;
        }
        if (at[i] < 0) t[i] = -CUDART_INF_F;
        here[i] = at[i] >= s.first && at[i] < s.first + s.count;
        z[i] = rank == 0 && at[i] >= 0 ? value_of(z_row[at[i]]) : 0.f;
    }
    load_share<T>(z_row, s, mem, [](const float (&)[P]) {});
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (here[i]) {
            const int pos = s.mis + at[i] - s.first;
            const uint32_t bit = 1u << (pos & 31);
            if (atomicOr(&named[pos >> 5], bit) & bit) sh.named_twice = 1;
            z[i] = value_of(z_mem[pos]);
        }
    __syncthreads();
    // an entry whose token an earlier one has already named: the first one stands for all of them
    bool stands[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) stands[i] = here[i];
    const bool twice = sh.named_twice != 0;
    if (twice)
        for (int i = 0; i < kMine; ++i)
            for (int k = 0; here[i] && k < threadIdx.x + i * kThreads; ++k)
                if (index[k] == at[i]) stands[i] = false;
    // ---- the student's sums
    const double scale = 1.4426950408889634 / (double)a.temperature;
    const float scale_f = (float)scale;
    auto words = [&](auto f) {
#pragma unroll 2
        for (int w = threadIdx.x; w < s.words; w += kThreads) {
            float x[P];
            unpack(mem[w], x);
            f(x, named[w * P >> 5] >> (w * P & 31));
        }
    };
    float mine = -CUDART_INF_F, sum = 0.f;
    words([&](const float (&x)[P], uint32_t marks) {
#pragma unroll
        for (int e = 0; e < P; ++e) mine = fmaxf(mine, marks >> e & 1 ? -CUDART_INF_F : x[e]);
    });
    const float from = mine == -CUDART_INF_F ? 0.f : mine;
    words([&](const float (&x)[P], uint32_t marks) {
#pragma unroll
        for (int e = 0; e < P; ++e) sum += exp2_fast(((marks >> e & 1 ? -CUDART_INF_F : x[e]) - from) * scale_f);
    });
    Sums own;
    own.top_others = over_cta(mine, larger, sh.scratch_f);
    own.others = over_cta((double)sum * rescale(mine, own.top_others, scale), add, sh.scratch);
    mine = -CUDART_INF_F;
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (stands[i]) mine = fmaxf(mine, z[i]);
    own.top_named = over_cta(mine, larger, sh.scratch_f);
    double part = 0.0;
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (stands[i] && z[i] != -CUDART_INF_F) part += rescale(z[i], own.top_named, scale);
    own.named = over_cta(part, add, sh.scratch);
    // ---- the teacher's softmax (in every CTA)
    const double T_ = (double)a.temperature;
    mine = -CUDART_INF_F;
#pragma unroll
    for (int i = 0; i < kMine; ++i) mine = fmaxf(mine, t[i]);
    const double top_t = fmax((double)over_cta(mine, larger, sh.scratch_f) / T_, (double)rest);
    part = threadIdx.x == 0 && rest != -CUDART_INF_F ? exp((double)rest - top_t) : 0.0;
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (t[i] != -CUDART_INF_F) part += exp((double)t[i] / T_ - top_t);
    const double log_t = top_t + log(over_cta(part, add, sh.scratch));
    begun_wait(a.ctas);
    int turn = 0;
    const Sums *all = tell(own, sh.told, turn, a.ctas, rank);
    float top_others = -CUDART_INF_F, top = -CUDART_INF_F;
    for (int c = 0; c < a.ctas; ++c) {
        top_others = fmaxf(top_others, all[c].top_others);
        top = fmaxf(top, all[c].top_named);
    }
    top = fmaxf(top, top_others);
    double others = 0.0, whole = 0.0;
    for (int c = 0; c < a.ctas; ++c) {
        others += all[c].others * rescale(all[c].top_others, top_others, scale);
        whole += all[c].named * rescale(all[c].top_named, top, scale);
    }
    whole += others * rescale(top_others, top, scale);
    if (whole == 0.0 || log_t == -CUDART_INF) {
        no_gradient();
        if (rank == 0 && threadIdx.x == 0) {
            a.loss[row] = 0.f;
            report(a.status, DSBD_DEV_EXHAUSTED);
        }
        return;
    }
    const double log_q = (double)top / T_ + log(whole);                 // of the student's sum
    const double log_others = (double)top_others / T_ + log(others) - log_q;
    const double p_rest = rest != -CUDART_INF_F ? exp((double)rest - log_t) : 0.0;
    // ---- the loss
    if (rank == 0) {
        part = threadIdx.x == 0 && p_rest != 0.0 ? p_rest * ((double)rest - log_t - log_others) : 0.0;
#pragma unroll
        for (int i = 0; i < kMine; ++i)
            if (t[i] != -CUDART_INF_F) {
                const double log_p = (double)t[i] / T_ - log_t, p = exp(log_p);
                if (p != 0.0) part += p * (log_p - ((double)z[i] / T_ - log_q));
            }
        part = over_cta(part, add, sh.scratch);
        if (threadIdx.x == 0) a.loss[row] = (float)(T_ * T_ * part);
    }
    if (!g_row) return;
    // ---- the gradient: the others', then the named tokens' over it
    const double unit = (double)weight * T_;
    double factor = 0.0;
    if (others != 0.0) factor = unit * (a.rest ? (exp(log_others) - p_rest) / others : rescale(top_others, top, scale) / whole);
    const float factor_f = (float)factor;
    const float base = top_others == -CUDART_INF_F ? 0.f : top_others;
    const bool along = ((reinterpret_cast<uintptr_t>(g_row + s.first) ^ reinterpret_cast<uintptr_t>(z_row + s.first)) & 15) == 0;
    put_share<T>(g_row, s, [&](int first, float (&g)[P]) {
        float x[P];
        if (along) {
            unpack(mem[(first + s.mis) / P], x);
        } else {
#pragma unroll
            for (int e = 0; e < P; ++e) x[e] = first + e >= 0 && first + e < s.count ? value_of(z_mem[s.mis + first + e]) : 0.f;
        }
#pragma unroll
        for (int e = 0; e < P; ++e) g[e] = factor_f * exp2_fast((x[e] - base) * scale_f);
    });
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (stands[i]) {
            double p = t[i] != -CUDART_INF_F ? exp((double)t[i] / T_ - log_t) : 0.0;
            if (twice)
                for (int k = threadIdx.x + i * kThreads + 1; k < a.K; ++k)
                    if (index[k] == at[i]) p += exp((double)value[k] / T_ - log_t);
            g_row[at[i]] = T((float)(unit * (exp((double)z[i] / T_ - log_q) - p)));
        }
}

}  // namespace
}  // namespace rows
}  // namespace dsbd

using namespace dsbd::rows;

extern "C" int dsbd_distill(const dsbd_rows_t *rows, const dsbd_distill_params_t *p, float *loss, void *grad, int64_t grad_stride,
                            int32_t *status, dsbd_stream_t stream) {
    int rc = check_rows(rows);
    if (rc) return rc;
    if (!p || p->K <= 0 || p->K > rows->V || !(p->temperature > 0.f && p->temperature <= FLT_MAX) || !status) return DSBD_ERR_INVALID_ARG;
    if (grad && rows->rows > 1 && grad_stride < rows->V) return DSBD_ERR_INVALID_ARG;
    const int size = rows->dtype == DSBD_DTYPE_F32 ? 4 : 2;
    if (p->K > DSBD_MAX_TOP || (reinterpret_cast<uintptr_t>(grad) & (size - 1))) return DSBD_ERR_UNSUPPORTED;
    if (rows->rows == 0) return DSBD_OK;
    if (!rows->logits || !p->value || !p->index || !loss) return DSBD_ERR_INVALID_ARG;
    const Plan plan = plan_for(rows);
    DistillArgs a = {};
    a.logits = rows->logits; a.stride = rows->row_stride; a.V = rows->V; a.K = p->K;
    a.ctas = plan.ctas; a.per = plan.per; a.words = plan.words; a.temperature = p->temperature;
    a.value = p->value; a.index = p->index; a.rest = p->rest; a.weight = p->weight;
    a.loss = loss; a.grad = grad; a.grad_stride = grad_stride; a.status = status;
    const size_t marks = ((size_t)plan.words * 16 / size / 32 + 1) * 4;
    return size == 4 ? launch(k_distill<float>, rows->rows, plan, marks, a, stream)
                     : launch(k_distill<__nv_bfloat16>, rows->rows, plan, marks, a, stream);
}
