// Verification of drafted tokens against the target's probabilities, from given random numbers.  Part of grpo.hip's
// translation unit.
//
//   p_i = softmax(z_i / T) of target row i, q_i the draft's (all on the drafted token where there are no draft logits)
//   draft y_i is accepted iff u_i q_i(y_i) < p_i(y_i), up to the first one, n, that is not
//   then one token: the smallest j with  sum_{l <= j} w_l > v sum_l w_l,  w = max(p_n - q_n, 0), or p_n behind the last draft
//
// Which token that is must not hang on the order in which 152064 terms are added up: with sums that are off by 1e-7 the
// border of some token lies between two orders' results in one row of a hundred.  So probabilities and sums are formed in fp64,
// in which that is one row in 10^8.
//
// A row is cut into `chunks` parts, each a workgroup's, so that a few rows fill the GPU too.  verify_rows_k forms each part's
// maximum and its sum of exponentials; verify_pick_k's workgroups, one to a part again, each find n from them, add up the
// part's w, and the last one of a response to do so finds the part in which the sum crosses v S, and in it the token.
// Behind the last draft w = p_n, whose sums are there already: one workgroup finds the token.

namespace __attribute__((visibility("hidden"))) grpo_impl {

constexpr int kVerifyBlock = 256;
constexpr int kMaxDrafts = 64;
constexpr int kMaxChunks = 1024;
constexpr int kVerifySlots = 8;  // vectors of a row that a lane holds at a time

struct VerifyPart {  // of a part of a row: its maximum, and the sum of exp((z - max) / T)
    double sum;
    float max;
    int pad;
};

struct Verify {
    const char *target, *draft;
    long long tb, tk, db, dk;  // pitches in bytes, of responses and of positions
    const long long *tokens;   // [batch][drafts]
    const float *u;            // [batch][drafts]
    const double *v;           // [batch]
    const int *lengths;
    int batch, drafts;
    long long vocab;
    int pickers;               // verify_pick_k's workgroups to a response: the parts, or 1 where nothing is drafted
    int chunks, chunk;         // parts of a row, and entries in one (of whole vectors of a whole workgroup)
    double k, kd;              // log2(e) / T, of the target and of the draft
    double inv_t;
    VerifyPart *part;          // [batch][2 drafts + 1][chunks]: target rows, then draft rows
    double *w;                 // [batch][chunks]: sums of the parts' w
    unsigned *ticket;          // [batch]
    long long *tokens_out;
    int *accepted_out;
    float *logprobs_out;

    __device__ __forceinline__ int length(int b) const
    {
        if (!lengths) return drafts;
        return lengths[b] < drafts ? lengths[b] : drafts;
    }
    __device__ __forceinline__ const char *target_row(int b, int i) const { return target + b * tb + i * tk; }
    __device__ __forceinline__ const char *draft_row(int b, int i) const { return draft + b * db + i * dk; }
    __device__ __forceinline__ const VerifyPart *parts(int b, int row) const { return part + ((long long)b * (2 * drafts + 1) + row) * chunks; }
};

// EPV entries of a row from entry j on, -inf behind its end.
template <grpo_dtype DT>
__device__ __forceinline__ void logits_load(const char *row, long long j, long long vocab, float (&z)[Elem<DT>::EPV])
{
    constexpr int EPV = Elem<DT>::EPV;
    if (j + EPV <= vocab) {
        unpack<DT>(*(const u32x4 *)(row + j * Elem<DT>::BYTES), z);
    } else {
#pragma unroll
        for (int i = 0; i < EPV; ++i) z[i] = j + i < vocab ? load_elem<DT>(row, j + i) : -INFINITY;
    }
}

// exp((z - m) / T) with k = log2(e) / T.  A sum is kept relative to a maximum m; where nothing has been added yet, or all of it is
// -inf, the maximum is -inf and 0 stands in for it in m's place: every z that is not NaN is -inf then and adds 0.
__device__ __forceinline__ double exp_from(float z, float m, double k)
{
    return exp2(((double)z - (double)m) * k);
}
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }

// A wavefront's lanes' (max, sum) pairs become the whole's in every lane.
__device__ __forceinline__ void wave_join(float &m, double &s, double k)
{
    const float top = wave_max(m);
    s = wave_sum_dpp(s * exp_from(m, finite_max(top), k));
    m = top;
}

template <grpo_dtype DT>
__global__ void __launch_bounds__(kVerifyBlock) verify_rows_k(Verify p)
{
    constexpr int EPV = Elem<DT>::EPV;
    __shared__ float lds_m[kVerifyBlock / 64];
    __shared__ double lds_s[kVerifyBlock / 64];
    const int c = blockIdx.x % p.chunks;
    const int rest = blockIdx.x / p.chunks;
    const int b = rest % p.batch, pos = rest / p.batch;  // positions in order, target and draft rows in turn
    const int i = p.draft ? pos >> 1 : pos;
    const bool drafted = p.draft && (pos & 1);
    const int len = p.length(b);
    if (pos == 0 && c == 0 && threadIdx.x == 0) p.ticket[b] = 0;
    if (drafted ? i >= len : i > len) return;
    const char *row = drafted ? p.draft_row(b, i) : p.target_row(b, i);
    const double k = drafted ? p.kd : p.k;
    const long long from = (long long)c * p.chunk, to = from + p.chunk < p.vocab ? from + p.chunk : p.vocab;
    float m = -INFINITY;
    double s = 0.0;
    for (long long j0 = from; j0 < to; j0 += kVerifyBlock * EPV * kVerifySlots) {
        float z[kVerifySlots][EPV];
        float top = m;
#pragma unroll
        for (int t = 0; t < kVerifySlots; ++t) logits_load<DT>(row, j0 + (t * kVerifyBlock + threadIdx.x) * EPV, to, z[t]);
#pragma unroll
        for (int t = 0; t < kVerifySlots; ++t)
#pragma unroll
            for (int e = 0; e < EPV; ++e) top = fmaxf(top, z[t][e]);
        top = wave_max(top);
        const float ref = finite_max(top);
        s *= exp_from(m, ref, k);
#pragma unroll
        for (int t = 0; t < kVerifySlots; ++t) {
            if (j0 + (long long)t * kVerifyBlock * EPV >= to) break;
#pragma unroll
            for (int e = 0; e < EPV; ++e) s += exp_from(z[t][e], ref, k);
        }
        m = top;
    }
    s = wave_sum_dpp(s);
    if ((threadIdx.x & 63) == 0) {
        lds_m[threadIdx.x >> 6] = m;
        lds_s[threadIdx.x >> 6] = s;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        float top = lds_m[0];
#pragma unroll
        for (int w = 1; w < kVerifyBlock / 64; ++w) top = fmaxf(top, lds_m[w]);
        s = 0.0;
#pragma unroll
        for (int w = 0; w < kVerifyBlock / 64; ++w) s += lds_s[w] * exp_from(lds_m[w], finite_max(top), k);
        VerifyPart *out = p.part + ((long long)b * (2 * p.drafts + 1) + (drafted ? p.drafts + 1 + i : i)) * p.chunks + c;
        out->max = top;
        out->sum = s;
    }
}

struct RowSum {
    double sum;
    float max;
};

// A row's maximum and sum from its parts', by one wavefront.
__device__ __forceinline__ RowSum row_sum(const VerifyPart *part, int chunks, double k)
{
    const int lane = threadIdx.x & 63;
    float m = -INFINITY;
    double s = 0.0;
    for (int c = lane; c < chunks; c += 64) {
        const VerifyPart q = part[c];
        const float top = fmaxf(m, q.max);
        s = s * exp_from(m, finite_max(top), k) + q.sum * exp_from(q.max, finite_max(top), k);
        m = top;
    }
    wave_join(m, s, k);
    return {s, m};
}

struct Residual {  // what w is made of
    const char *t, *d;  // target row, draft row (NULL: the draft has all of its mass on token y, or there is none: y = -1)
    long long y;
    double k, kd, inv_sp, inv_sq;
    float mp, mq;
};

// w of EPV entries from entry j on.
template <grpo_dtype DT>
__device__ __forceinline__ void weights(const Residual &r, long long j, long long vocab, double (&w)[Elem<DT>::EPV])
{
#pragma clang fp contract(off)  // equal rows leave 0, not the rounding of one of the two products
    constexpr int EPV = Elem<DT>::EPV;
    float z[EPV];
    logits_load<DT>(r.t, j, vocab, z);
#pragma unroll
    for (int e = 0; e < EPV; ++e) w[e] = exp_from(z[e], r.mp, r.k) * r.inv_sp;
    if (r.d) {
        logits_load<DT>(r.d, j, vocab, z);
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
            w[e] -= exp_from(z[e], r.mq, r.kd) * r.inv_sq;
            if (w[e] < 0.0) w[e] = 0.0;  // NaN stays
        }
    } else {
#pragma unroll
        for (int e = 0; e < EPV; ++e)
            if (j + e == r.y) w[e] = w[e] == w[e] ? 0.0 : w[e];
    }
}

__device__ __forceinline__ double wave_scan(double v)  // sums of the lanes up to and with this one
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double up = __shfl_up(v, o, 64);
        if (lane >= o) v += up;
    }
    return v;
}

struct PickLds {
    double prefix[kMaxChunks];
    double wave[kVerifyBlock / 64];
    int part, found, last;
    long long token;
};

// The token: the parts' sums are in lds.prefix.  -1 where they have no sum, or it is no number.  All lanes take part and get it.
template <grpo_dtype DT>
__device__ long long pick_token(const Verify &p, const Residual &r, double v, PickLds &lds)
{
    constexpr int EPV = Elem<DT>::EPV;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (tid == 0) {
        lds.part = 0x7fffffff;
        lds.last = -1;
    }
    __syncthreads();
    double total = 0.0;
    if (wave == 0) {
        int last = -1;
        for (int c0 = 0; c0 < p.chunks; c0 += 64) {
            const int c = c0 + lane;
            const double w = c < p.chunks ? lds.prefix[c] : 0.0;
            if (w > 0.0) last = c;
            const double up = total + wave_scan(w);
            if (c < p.chunks) lds.prefix[c] = up;
            total = __shfl(up, 63, 64);
        }
        atomicMax(&lds.last, last);
    }
    __syncthreads();
    total = lds.prefix[p.chunks - 1];
    if (!(total > 0.0) || !(total < INFINITY)) return -1;
    const double target = v * total;
    for (int c = tid; c < p.chunks; c += kVerifyBlock)
        if (lds.prefix[c] > target) {
            atomicMin(&lds.part, c);
            break;
        }
    __syncthreads();
    // a number next to 1 times the sum may be the sum: then the last token that has any
    const int c = lds.part < p.chunks ? lds.part : lds.last;
    __syncthreads();
    if (tid == 0) lds.last = -1;
    double base = c > 0 ? lds.prefix[c - 1] : 0.0;
    const long long from = (long long)c * p.chunk, to = from + p.chunk < p.vocab ? from + p.chunk : p.vocab;
    int fallback = -1;  // of this lane: its last entry with a weight
    for (long long j0 = from; j0 < to; j0 += kVerifyBlock * EPV) {
        const long long j = j0 + tid * EPV;
        double w[EPV], sum = 0.0;
        weights<DT>(r, j, to, w);
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
            sum += w[e];
            if (w[e] > 0.0) fallback = (int)(j - from) + e;
        }
        const double up = wave_scan(sum);
        if (lane == 63) lds.wave[wave] = up;
        if (tid == 0) lds.found = 0x7fffffff;
        __syncthreads();
        double before = base;
#pragma unroll
        for (int i = 0; i < kVerifyBlock / 64; ++i) {
            if (i < wave) before += lds.wave[i];
            base += lds.wave[i];
        }
        if (before + up > target) atomicMin(&lds.found, tid);
        __syncthreads();
        if (lds.found == tid) {  // the first lane whose entries cross; one of them does, up to rounding
            double run = before + (up - sum);
            int at = fallback;
#pragma unroll
            for (int e = EPV - 1; e >= 0; --e) {
                double s = run;
#pragma unroll
                for (int i = 0; i <= e; ++i) s += w[i];
                if (s > target && w[e] > 0.0) at = (int)(j - from) + e;
            }
            lds.token = from + at;
        }
        __syncthreads();
        if (lds.found < kVerifyBlock) return lds.token;
        __syncthreads();
    }
    // the part's entries, added up in another order, stay below what its sum promised: the last that has any
    atomicMax(&lds.last, fallback);
    __syncthreads();
    return from + lds.last;
}

template <grpo_dtype DT>
__global__ void __launch_bounds__(kVerifyBlock) verify_pick_k(Verify p)
{
    constexpr int EPV = Elem<DT>::EPV;
    __shared__ double ratio_p[kMaxDrafts], ratio_q[kMaxDrafts];
    __shared__ RowSum row_p[kMaxDrafts + 1], row_q[kMaxDrafts];
    __shared__ PickLds lds;
    __shared__ bool last_one;
    const int b = blockIdx.x / p.pickers, c = blockIdx.x % p.pickers;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int len = p.length(b);
    const int K = p.drafts;
    long long *tokens_out = p.tokens_out + (long long)b * (K + 1);
    float *logprobs_out = p.logprobs_out + (long long)b * (K + 1);
    if (len < 0) {  // not a response
        if (c == 0) {
            for (int i = tid; i <= K; i += kVerifyBlock) {
                tokens_out[i] = -1;
                logprobs_out[i] = 0.f;
            }
            if (tid == 0) p.accepted_out[b] = 0;
        }
        return;
    }
    for (int i = wave; i <= len; i += kVerifyBlock / 64) {
        const RowSum rp = row_sum(p.parts(b, i), p.chunks, p.k);
        RowSum rq = {1.0, 0.f};
        if (p.draft && i < len) rq = row_sum(p.parts(b, K + 1 + i), p.chunks, p.kd);
        if (lane == 0) {
            row_p[i] = rp;
            if (i < len) {
                row_q[i] = rq;
                const long long y = p.tokens[(long long)b * K + i];
                const bool in = y >= 0 && y < p.vocab;
                ratio_p[i] = in ? exp_from(load_elem<DT>(p.target_row(b, i), y), rp.max, p.k) / rp.sum : 0.0;
                ratio_q[i] = !p.draft ? 1.0 : in ? exp_from(load_elem<DT>(p.draft_row(b, i), y), rq.max, p.kd) / rq.sum : 0.0;
            }
        }
    }
    __syncthreads();
    int n = 0;
    while (n < len && (double)p.u[(long long)b * K + n] * ratio_q[n] < ratio_p[n]) ++n;
    if (c == 0) {
        for (int i = tid; i <= K; i += kVerifyBlock) {
            if (i < n) {
                tokens_out[i] = p.tokens[(long long)b * K + i];
                logprobs_out[i] = (float)log(ratio_p[i]);
            } else if (i > n) {
                tokens_out[i] = -1;
                logprobs_out[i] = 0.f;
            }
        }
        if (tid == 0) p.accepted_out[b] = n;
    }
    Residual r = {};
    r.t = p.target_row(b, n);
    r.y = -1;
    r.k = p.k;
    r.kd = p.kd;
    r.mp = row_p[n].max;
    r.inv_sp = 1.0;
    bool residual = n < len;
    if (residual) {
        r.inv_sp = 1.0 / row_p[n].sum;
        if (p.draft) {
            r.d = p.draft_row(b, n);
            r.mq = row_q[n].max;
            r.inv_sq = 1.0 / row_q[n].sum;
        } else {
            r.y = p.tokens[(long long)b * K + n];
        }
        const long long from = (long long)c * p.chunk, to = from + p.chunk < p.vocab ? from + p.chunk : p.vocab;
        double s = 0.0;
        for (long long j = from + tid * EPV; j < to; j += kVerifyBlock * EPV) {
            double w[EPV];
            weights<DT>(r, j, to, w);
#pragma unroll
            for (int e = 0; e < EPV; ++e) s += w[e];
        }
        s = wave_sum_dpp(s);
        if (lane == 0) lds.wave[wave] = s;
        __syncthreads();
        if (tid == 0) {
            s = 0.0;
#pragma unroll
            for (int i = 0; i < kVerifyBlock / 64; ++i) s += lds.wave[i];
            p.w[(long long)b * p.chunks + c] = s;
            __threadfence();
            last_one = atomicAdd(&p.ticket[b], 1u) == (unsigned)p.chunks - 1;
        }
        __syncthreads();
        if (!last_one) return;
        __threadfence();
        for (int i = tid; i < p.chunks; i += kVerifyBlock) lds.prefix[i] = p.w[(long long)b * p.chunks + i];
    } else {
        if (c != 0) return;
    }
    long long token = -1;
    __syncthreads();
    for (int pass = residual ? 0 : 1; pass < 2; ++pass) {
        if (pass == 1) {
            // behind the last draft, or with nothing left of p - q but rounding: from p itself
            r.d = nullptr;
            r.y = -1;
            r.inv_sp = 1.0;
            const VerifyPart *part = p.parts(b, n);
            for (int i = tid; i < p.chunks; i += kVerifyBlock)
                lds.prefix[i] = part[i].sum * exp_from(part[i].max, finite_max(r.mp), p.k);
        }
        __syncthreads();
        token = pick_token<DT>(p, r, p.v[b], lds);
        const bool nothing = lds.prefix[p.chunks - 1] == 0.0;
        __syncthreads();
        if (!nothing) break;
    }
    if (tid == 0) {
        tokens_out[n] = token;
        logprobs_out[n] = token < 0 ? __builtin_nanf("")
                                    : (float)(((double)load_elem<DT>(r.t, token) - (double)r.mp) * p.inv_t - log(row_p[n].sum));
    }
}

// Entries in a part of a row, and parts.  Enough parts that all rows' fill the GPU, and no more than pick_token has room for.
static bool verify_plan(int64_t batch, int64_t drafts, int64_t vocab, int dtype, int *chunk, int *chunks)
{
    if (batch < 0 || batch > 0x7fffffffll || drafts < 0 || drafts > kMaxDrafts || vocab <= 0 || vocab > kMaxVocab) return false;
    const int64_t rows = batch * (2 * drafts + 1);
    const int64_t unit = kVerifyBlock * (dtype == GRPO_BF16 ? 8 : 4);
    int64_t units = 1;
    while ((vocab + units * unit - 1) / (units * unit) > kMaxChunks) units *= 2;
    while (units < kVerifySlots && rows * ((vocab + unit * units - 1) / (unit * units)) >= 4096) units *= 2;
    *chunk = (int)(units * unit);
    *chunks = (int)((vocab + units * unit - 1) / (units * unit));
    return rows * *chunks <= 0x7fffffffll;  // workgroups
}

}  // namespace grpo_impl

extern "C" {

size_t grpo_verify_workspace_bytes(int64_t batch, int64_t drafts, int64_t vocab, grpo_dtype dtype_arg)
{
    const int dtype = raw_enum(dtype_arg);
    int chunk, chunks;
    if ((dtype != GRPO_F32 && dtype != GRPO_BF16) || !verify_plan(batch, drafts, vocab, dtype, &chunk, &chunks)) return 0;
    return align_up((size_t)batch * 4 + 1, 256) + align_up((size_t)batch * chunks * 8, 256) +
           (size_t)batch * (2 * drafts + 1) * chunks * sizeof(VerifyPart);
}

grpo_status grpo_verify_drafts(const void *target_logits, int64_t target_batch_stride, int64_t target_row_stride, const void *draft_logits,
                               int64_t draft_batch_stride, int64_t draft_row_stride, grpo_dtype dtype_arg, int64_t batch, int64_t drafts,
                               int64_t vocab, const int64_t *draft_tokens, const float *accept_u, const double *sample_u,
                               const int32_t *draft_lengths, double temperature, double draft_temperature, int64_t *tokens_out,
                               int32_t *n_accepted_out, float *logprobs_out, void *workspace, size_t workspace_bytes, void *stream)
{
    const int dtype = raw_enum(dtype_arg);
    if (dtype != GRPO_F32 && dtype != GRPO_BF16) return GRPO_ERR_DTYPE;
    Verify p = {};
    if (!verify_plan(batch, drafts, vocab, dtype, &p.chunk, &p.chunks)) return GRPO_ERR_SHAPE;
    if (!(temperature > 0.0) || !std::isfinite(temperature) || !(draft_temperature > 0.0) || !std::isfinite(draft_temperature)) return GRPO_ERR_PARAM;
    if (batch == 0) return GRPO_OK;
    if (!target_logits || !sample_u || !tokens_out || !n_accepted_out || !logprobs_out) return GRPO_ERR_NULL;
    if (drafts > 0 && (!draft_tokens || !accept_u)) return GRPO_ERR_NULL;
    if (drafts == 0) draft_logits = nullptr;
    const int64_t bytes = dtype == GRPO_BF16 ? 2 : 4;
    if (target_row_stride < vocab || target_batch_stride < 0 || (draft_logits && (draft_row_stride < vocab || draft_batch_stride < 0)))
        return GRPO_ERR_SHAPE;
    if (((uintptr_t)target_logits & 15u) || ((target_row_stride * bytes) & 15) || ((target_batch_stride * bytes) & 15)) return GRPO_ERR_ALIGN;
    if (draft_logits && (((uintptr_t)draft_logits & 15u) || ((draft_row_stride * bytes) & 15) || ((draft_batch_stride * bytes) & 15)))
        return GRPO_ERR_ALIGN;
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < grpo_verify_workspace_bytes(batch, drafts, vocab, dtype_arg))
        return GRPO_ERR_WORKSPACE;
    p.target = (const char *)target_logits;
    p.tb = target_batch_stride * bytes;
    p.tk = target_row_stride * bytes;
    p.draft = (const char *)draft_logits;
    p.db = draft_batch_stride * bytes;
    p.dk = draft_row_stride * bytes;
    p.tokens = (const long long *)draft_tokens;
    p.u = accept_u;
    p.v = sample_u;
    p.lengths = draft_lengths;
    p.batch = (int)batch;
    p.drafts = (int)drafts;
    p.vocab = vocab;
    const double log2e = 1.4426950408889634074;
    p.inv_t = 1.0 / temperature;
    p.k = log2e / temperature;
    p.kd = log2e / draft_temperature;
    char *ws = (char *)workspace;
    p.ticket = (unsigned *)ws;
    ws += align_up((size_t)batch * 4 + 1, 256);
    p.w = (double *)ws;
    ws += align_up((size_t)batch * p.chunks * 8, 256);
    p.part = (VerifyPart *)ws;
    p.tokens_out = (long long *)tokens_out;
    p.accepted_out = n_accepted_out;
    p.logprobs_out = logprobs_out;
    hipStream_t st = (hipStream_t)stream;
    const unsigned row_blocks = (unsigned)(batch * (draft_logits ? 2 * drafts + 1 : drafts + 1) * p.chunks);
    p.pickers = drafts > 0 ? p.chunks : 1;
    const unsigned pick_blocks = (unsigned)(batch * p.pickers);
    if (dtype == GRPO_BF16) {
        hipLaunchKernelGGL(verify_rows_k<GRPO_BF16>, dim3(row_blocks), dim3(kVerifyBlock), 0, st, p);
        hipLaunchKernelGGL(verify_pick_k<GRPO_BF16>, dim3(pick_blocks), dim3(kVerifyBlock), 0, st, p);
    } else {
        hipLaunchKernelGGL(verify_rows_k<GRPO_F32>, dim3(row_blocks), dim3(kVerifyBlock), 0, st, p);
        hipLaunchKernelGGL(verify_pick_k<GRPO_F32>, dim3(pick_blocks), dim3(kVerifyBlock), 0, st, p);
    }
    return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}

}  // extern "C"
