// The largest logits of rows, with the log-sum-exp of the rest.
#include "dsbd_top.cuh"

namespace dsbd {
namespace rows {
namespace {

struct TopArgs {
    const void *logits;
    int64_t stride;
    int V, K, ctas, per;
    float temperature;
    float *value;
    int32_t *index;
    float *rest;
    int32_t *status;
};

struct Part {
    Sum rest;
    uint32_t listed;                               // ~0: a NaN or +inf
};

// A row is one CTA's (a cluster's where there are few): it streams its share once and at the end sorts little more than K entries.  Long
// rows are bound by HBM (4608 rows of 128256 fp32, K = 64: 464 us, 5.1 TB/s, of 362 at the copy rate; from one GPU to another up to 485); short ones with many entries by the
// instructions that a row needs however short it is -- bounds, sorting kept words out, the list's order: 2048 rows of 32000 bf16,
// K = 256: 125 us for 21 of bytes, 39 thousand warp instructions a row.  Small CTAs, many on an SM, let some rows stream
// while others sort (128 threads 124 us, 256 140, 512 192).  A few rows are a chain of load, bounds, exchange and sort: 20 rows of 50257, 15 us.
template <class T, int NT, int G, int LIST, int HOT, int CTAS>
__global__ void __launch_bounds__(NT, CTAS) k_top(TopArgs a) {
    using L = TopList<NT, G, LIST, HOT>;
    extern __shared__ float4 mem[];
    L &sh = *reinterpret_cast<L *>(mem);
    __shared__ Told<Part> told;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    begun_arrive(a.ctas);
    const int row = blockIdx.x / a.ctas, rank = blockIdx.x - row * a.ctas;
    const T *at = static_cast<const T *>(a.logits) + (int64_t)row * a.stride;
    float *value_out = a.value + (int64_t)row * a.K;
    int32_t *index_out = a.index + (int64_t)row * a.K;
    const double scale = 1.4426950408889634 / (double)a.temperature;
    const float scale_f = (float)scale;
    Rest rest;
    Sum cleared = {-CUDART_INF_F, 0.0};
    const bool good = collect<T, true>(sh, at, share<T>(at, a.V, rank, a.per), (uint32_t)a.K, a.ctas > 1, scale_f, rest, cleared);
    // the threads' sums and what was cleared
    auto joined = [&] {
        Sum s = {rest.high, 0.0};
        float low = 0.f;
        sh.range(s.high, low);
        const double d = warp_sum((double)rest.sum * rescale(rest.high, s.high, scale));
        if ((threadIdx.x & 31) == 0) sh.sums[threadIdx.x / 32] = d;
        __syncthreads();
        for (int w = 0; w < NT / 32; ++w) s.sum += sh.sums[w];
        s.add(cleared, scale);
        return s;
    };
    const Part own = {joined(), good ? sh.listed : ~0u};
    begun_wait(a.ctas);
    int turn = 0;
    const Part *all = tell(own, told, turn, a.ctas, rank);
    bool bad = false;
    uint64_t n = 0;
    for (int c = 0; c < a.ctas; ++c) {
        bad |= all[c].listed == ~0u;
        n += all[c].listed;
    }
    const bool over = n > LIST;
    if (rank == 0 && !bad && !over) {
        uint32_t to = own.listed;
        for (int c = 1; c < a.ctas; ++c) {
            const uint64_t *from = cg::this_cluster().map_shared_rank(&sh.list[0], c);
            for (uint32_t i = threadIdx.x; i < all[c].listed; i += NT) sh.list[to + i] = from[i];
            to += all[c].listed;
        }
        if (threadIdx.x == 0) sh.listed = to;
    }
    cluster_barrier(a.ctas);                       // (rank 0 has the lists)
    if (rank) return;
    if (bad || n == 0) {
        for (int i = threadIdx.x; i < a.K; i += NT) {
            value_out[i] = CUDART_NAN_F;
            index_out[i] = -1;
        }
        if (threadIdx.x == 0) {
            if (a.rest) a.rest[row] = CUDART_NAN_F;
            report(a.status, bad ? DSBD_DEV_BAD_LOGIT : DSBD_DEV_EXHAUSTED);
        }
        return;
    }
    rest = Rest();
    cleared = {-CUDART_INF_F, 0.0};
    if (over) {
        select_row<T, true>(sh, at, a.V, (uint32_t)a.K, scale_f, rest);
    } else {
        for (int c = 0; c < a.ctas; ++c) cleared.add(all[c].rest, scale);
        sh.template clear<true>(sh.entries_bound((uint32_t)a.K), scale_f, cleared);
    }
    sh.sort();
    const int kept = min((int)sh.listed, a.K);
    for (int i = threadIdx.x; i < (int)sh.listed; i += NT) {
        if (i < kept) {
            value_out[i] = logit_of(sh.list[i]);
            index_out[i] = token_of(sh.list[i]);
        } else {
            rest.add(logit_of(sh.list[i]), scale_f);
        }
    }
    if (a.rest) {
        const Sum s = joined();
        if (threadIdx.x == 0) a.rest[row] = s.sum > 0.0 ? (float)((double)s.high / (double)a.temperature + log(s.sum)) : -CUDART_INF_F;
    }
    if (threadIdx.x < 32)
        // fewer than K above -inf: the first tokens at -inf
        for (int t0 = 0, to0 = kept; to0 < a.K && t0 < a.V; t0 += 32) {
            const int t = t0 + threadIdx.x;
            const unsigned m = __ballot_sync(kFull, t < a.V && value_of(at[min(t, a.V - 1)]) == -CUDART_INF_F);
            const int to = to0 + __popc(m & ((1u << threadIdx.x) - 1));
            if ((m >> threadIdx.x & 1) && to < a.K) {
                value_out[to] = -CUDART_INF_F;
                index_out[to] = t;
            }
            to0 += __popc(m);
        }
}

// CTAs of a row: as many as run at once (resident ones of an SM), none with less than half a batch, and lists that fit into one.  (More CTAs
// of a row than run at once, to even out the waves, cost what a CTA does for each row: 592 rows of 128256 91 us, in two CTAs each 108.)
inline Plan plan_top(const dsbd_rows_t *r, int threads, int resident, int list, int K) {
    Plan p = {1, 0, 0};
    while (p.ctas < kMaxCtas && r->rows * 2 * (int64_t)p.ctas <= 148 * resident && share_of(r->V, 2 * p.ctas) >= threads * 16 &&
           3 * (int64_t)K * p.ctas <= list)
        p.ctas *= 2;
    p.per = share_of(r->V, p.ctas);
    return p;
}

template <class T, int NT, int G, int LIST, int HOT, int CTAS>
int run_top(const dsbd_rows_t *r, TopArgs &a, dsbd_stream_t stream) {
    const Plan p = plan_top(r, NT, CTAS, LIST, a.K);
    a.ctas = p.ctas;
    a.per = p.per;
    return launch<sizeof(TopList<NT, G, LIST, HOT>), NT>(k_top<T, NT, G, LIST, HOT, CTAS>, r->rows, p, sizeof(TopList<NT, G, LIST, HOT>), a, stream);
}

}  // namespace
}  // namespace rows
}  // namespace dsbd

using namespace dsbd::rows;

extern "C" int dsbd_top_logits(const dsbd_rows_t *rows, int32_t K, float temperature, float *value, int32_t *index, float *rest,
                               int32_t *status, dsbd_stream_t stream) {
    int rc = check_rows(rows);
    if (rc) return rc;
    if (K <= 0 || K > rows->V || !scales(temperature) || !status) return DSBD_ERR_INVALID_ARG;
    if (K > DSBD_MAX_TOP) return DSBD_ERR_UNSUPPORTED;
    if (rows->rows == 0) return DSBD_OK;
    if (!rows->logits || !value || !index) return DSBD_ERR_INVALID_ARG;
    TopArgs a = {};
    a.logits = rows->logits; a.stride = rows->row_stride; a.V = rows->V; a.K = K; a.temperature = temperature;
    a.value = value; a.index = index; a.rest = rest; a.status = status;
    // Where there are rows enough, small CTAs: what a CTA does once for each row costs fewer instructions (4608 rows of 128256 465 us,
    // with 256 threads 496; 512 rows 85 and 88; 296 rows 57 and 52)
    if (K <= 256 && rows->rows >= 148 * 3)
        return rows->dtype == DSBD_DTYPE_F32 ? run_top<float, 128, 4, 1024, 1024, 6>(rows, a, stream)
                                             : run_top<__nv_bfloat16, 128, 4, 1024, 1024, 6>(rows, a, stream);
    if (K <= 512)
        return rows->dtype == DSBD_DTYPE_F32 ? run_top<float, 256, 4, 2048, 1536, 3>(rows, a, stream)
                                             : run_top<__nv_bfloat16, 256, 4, 2048, 1536, 3>(rows, a, stream);
    return rows->dtype == DSBD_DTYPE_F32 ? run_top<float, 512, 4, 4096, 2560, 2>(rows, a, stream)
                                         : run_top<__nv_bfloat16, 512, 4, 4096, 2560, 2>(rows, a, stream);
}
