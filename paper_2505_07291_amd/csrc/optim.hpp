// What a trainer does with the gradients: their norm over all tensors (section 4.1 of the paper clips it at 0.1) and one AdamW
// step.  Part of grpo.hip's translation unit.
//
//   norm = sqrt(sum over all tensors of g^2),  coefficient = norm <= max_norm ? 1 : max_norm / norm
//   g' = coefficient g
//   m  = beta1 m + (1 - beta1) g'          v = beta2 v + (1 - beta2) g'^2
//   p  = p (1 - lr wd) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// Both walk over a table in device memory, made once by grpo_optim_plan_build: the tensors, and for every 4096 values of
// them which tensor and which 4096 (a look-up by a value's index would be ten dependent loads with a thousand tensors).  So a
// model of any number of tensors is one launch, whose workgroups all have the same work.
//
// Values are taken 256 at a time by a wavefront, which are also the 256 that share a scale of the 8-bit moments: four
// neighbours to a lane (16-byte accesses of fp32) where the tensor's arrays begin on 16-byte boundaries, four that are 64 apart
// (4-byte accesses, still whole lines to a wavefront) where one does not, or where the tensor ends inside the 256.

namespace __attribute__((visibility("hidden"))) grpo_impl {

struct OptTensor {
    void *param;
    float *master;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale;
    long long n;
    double weight_decay;
    int param_bf16, grad_bf16, state8, wide;  // wide: every array begins on a boundary of four values' 16, 8 or 4 bytes
};
static_assert(sizeof(OptTensor) == 88, "the table's entries lie behind one another");
struct OptChunk {
    int tensor, chunk;
};

constexpr int kOptBlock = 256;
constexpr long long kMaxWorkgroups = 0xffffffffll / kOptBlock;  // a launch has less than 2^32 lanes
constexpr int kOptQuant = 256;    // values to a scale, and to a wavefront's step
constexpr int kOptChunk = 4096;   // values to a workgroup of adamw_step_k
constexpr long long kOptMaxValues = 1ll << 40;  // of one tensor
constexpr int kNormBlocks = 2048; // workgroups, and partial sums, of grad_norm_k

constexpr size_t opt_chunks_at(long long n_tensors) { return ((size_t)n_tensors * sizeof(OptTensor) + 255) / 256 * 256; }

struct AdamW {
    const OptTensor *tensors;
    const OptChunk *chunks;
    const float *clip;           // clip[1]: the coefficient; or NULL
    const float *lr_at;          // the learning rate and the step's number, where they are in device memory
    const long long *step_at;
    double lr, log_beta1, log_beta2;
    double bias1;                // 1 - beta1^t and 1 / sqrt(1 - beta2^t), where the step's number comes from the host
    float inv_root;
    float beta1, one_beta1, beta2, one_beta2, eps;
};

__device__ __forceinline__ float bf16_to_f32(unsigned short u) { return as_f32((unsigned)u << 16); }
__device__ __forceinline__ unsigned bf16_pair(float a, float b)
{
    const f32x2 p = {a, b};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(p, bf16x2));
}

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// Four values of a wavefront's 256: neighbours at 4 lane (WIDE), or the ones at lane + 64 j below `left`.
template <bool WIDE>
__device__ __forceinline__ void load4_f32(const float *p, int lane, int left, float (&x)[4])
{
    if constexpr (WIDE) {
        const u32x4 v = ld16((const char *)(p + 4 * lane));
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = as_f32(v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = lane + 64 * j < left ? p[lane + 64 * j] : 0.f;
    }
}
template <bool WIDE>
__device__ __forceinline__ void load4_bf16(const unsigned short *p, int lane, int left, float (&x)[4])
{
    if constexpr (WIDE) {
        const u32x2 v = __builtin_nontemporal_load((const u32x2 *)(p + 4 * lane));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            x[2 * j] = as_f32(v[j] << 16);
            x[2 * j + 1] = as_f32(v[j] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = lane + 64 * j < left ? bf16_to_f32(p[lane + 64 * j]) : 0.f;
    }
}
template <bool WIDE>
__device__ __forceinline__ void store4_f32(float *p, int lane, int left, const float (&x)[4])
{
    if constexpr (WIDE) {
        const u32x4 v = {as_u32(x[0]), as_u32(x[1]), as_u32(x[2]), as_u32(x[3])};
        st16((char *)(p + 4 * lane), v);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (lane + 64 * j < left) p[lane + 64 * j] = x[j];
    }
}
template <bool WIDE>
__device__ __forceinline__ void store4_bf16(unsigned short *p, int lane, int left, const float (&x)[4])
{
    const u32x2 v = {bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
    if constexpr (WIDE) {
        __builtin_nontemporal_store(v, (u32x2 *)(p + 4 * lane));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (lane + 64 * j < left) p[lane + 64 * j] = (unsigned short)(v[j >> 1] >> (16 * (j & 1)));
    }
}

// Moments in 8 bits: e4m3 codes times a power of two to 256 values, the least one under which the largest of them is at
// most 448.  A power of two costs up to a bit of e4m3's range (not of its precision) and makes both scalings exact, so that a
// value is rounded once.  What is not finite becomes NaN and does not count for the scale: its neighbours stay.
template <bool WIDE>
__device__ __forceinline__ void load4_e4m3(const unsigned char *p, int lane, int left, float scale, float (&x)[4])
{
    unsigned w = 0;
    if constexpr (WIDE) {
        w = __builtin_nontemporal_load((const unsigned *)(p + 4 * lane));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (lane + 64 * j < left) w |= (unsigned)p[lane + 64 * j] << (8 * j);
    }
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0] * scale;
    x[1] = lo[1] * scale;
    x[2] = hi[0] * scale;
    x[3] = hi[1] * scale;
}
// KEEP: a positive value becomes at least the smallest code (a second moment of 0 under a first moment that is not would
// make a step of m / eps).
template <bool WIDE, bool KEEP>
__device__ __forceinline__ void store4_e4m3(unsigned char *p, float *scale_out, int lane, int left, const float (&x)[4])
{
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = fmaxf(top, fabsf(x[j]) < INFINITY ? fabsf(x[j]) : 0.f);
    const unsigned bits = as_u32(wave_max(top));
    int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    if (e < -126) e = -126;
    const float inv = as_f32((unsigned)(127 - e) << 23);
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        y[j] = x[j] * inv;
        if (KEEP && x[j] > 0.f) y[j] = fmaxf(y[j], 0x1p-9f);
        if (!(fabsf(y[j]) <= 448.f)) y[j] = __builtin_nanf("");
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
    if constexpr (WIDE) {
        __builtin_nontemporal_store((unsigned)w, (unsigned *)(p + 4 * lane));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (lane + 64 * j < left) p[lane + 64 * j] = (unsigned char)((unsigned)w >> (8 * j));
    }
    if (lane == 0) *scale_out = as_f32((unsigned)(e + 127) << 23);
}

enum { kParamF32 = 0, kParamBf16 = 1, kParamMaster = 2 };  // kParamMaster: bf16, written from the fp32 master copy

struct AdamWStep {  // the same for a whole workgroup
    float coef, decay, step_size, inv_root;
};

// U times 256 values of a tensor, from value `at` on and every `step`; of the last 256 `left` are there.  Everything is asked for
// before anything is written: the compiler cannot move a load in front of a store.
template <int PARAM, bool GBF16, bool STATE8, bool WIDE, int U>
__device__ __forceinline__ void adamw_256(const AdamW &a, const AdamWStep &s, const OptTensor &t, long long at, int step, int left, int lane)
{
    float g[U][4], m[U][4], v[U][4], p[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long i = at + u * step, block = i / kOptQuant;
        if constexpr (GBF16)
            load4_bf16<WIDE>((const unsigned short *)t.grad + i, lane, left, g[u]);
        else
            load4_f32<WIDE>((const float *)t.grad + i, lane, left, g[u]);
        if constexpr (STATE8) {
            load4_e4m3<WIDE>((const unsigned char *)t.m + i, lane, left, t.m_scale[block], m[u]);
            load4_e4m3<WIDE>((const unsigned char *)t.v + i, lane, left, t.v_scale[block], v[u]);
        } else {
            load4_f32<WIDE>((const float *)t.m + i, lane, left, m[u]);
            load4_f32<WIDE>((const float *)t.v + i, lane, left, v[u]);
        }
        if constexpr (PARAM == kParamF32)
            load4_f32<WIDE>((const float *)t.param + i, lane, left, p[u]);
        else if constexpr (PARAM == kParamBf16)
            load4_bf16<WIDE>((const unsigned short *)t.param + i, lane, left, p[u]);
        else
            load4_f32<WIDE>(t.master + i, lane, left, p[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long i = at + u * step, block = i / kOptQuant;
        float r[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // Every operation is rounded by itself, in this order: what a step gives does not hang on which sums the compiler
            // fuses, and 8-bit moments are rounded from values that anybody can compute again.
#pragma clang fp contract(off)
            const float gc = g[u][j] * s.coef;
            if constexpr (STATE8) v[u][j] = v[u][j] * v[u][j];  // sqrt(v) is what is held
            m[u][j] = m[u][j] * a.beta1 + gc * a.one_beta1;
            v[u][j] = v[u][j] * a.beta2 + gc * gc * a.one_beta2;
            r[j] = __builtin_sqrtf(v[u][j]);
            const float move = m[u][j] / (r[j] * s.inv_root + a.eps);
            p[u][j] = p[u][j] * s.decay - move * s.step_size;
        }
        if constexpr (PARAM != kParamF32) store4_bf16<WIDE>((unsigned short *)t.param + i, lane, left, p[u]);
        if constexpr (PARAM == kParamF32) store4_f32<WIDE>((float *)t.param + i, lane, left, p[u]);
        if constexpr (PARAM == kParamMaster) store4_f32<WIDE>(t.master + i, lane, left, p[u]);
        if constexpr (STATE8) {
            store4_e4m3<WIDE, false>((unsigned char *)t.m + i, t.m_scale + block, lane, left, m[u]);
            store4_e4m3<WIDE, true>((unsigned char *)t.v + i, t.v_scale + block, lane, left, r);
        } else {
            store4_f32<WIDE>((float *)t.m + i, lane, left, m[u]);
            store4_f32<WIDE>((float *)t.v + i, lane, left, v[u]);
        }
    }
}

// 256s that a wavefront asks for at a time.  123 million values with 8-bit moments take 345 us by four, 364 by two and 374 one by one, and
// 338 where those four are all a workgroup does (kOptChunk; at 16384 370); 778 million with fp32 moments and a master copy
// 4.32 ms and 4.18 (5.6 TB/s).  Loads or stores that may stay in the caches cost 3 to 9 %.
constexpr int kOptAhead = 4;
template <int PARAM, bool GBF16, bool STATE8>
__device__ __forceinline__ void adamw_chunk(const AdamW &a, const AdamWStep &s, const OptTensor &t, long long first)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int kStep = kOptBlock / 64 * kOptQuant;
    if (t.wide && t.n - first >= kOptChunk) {
#pragma unroll 1
        for (int i = 0; i < kOptChunk; i += kOptAhead * kStep)
            adamw_256<PARAM, GBF16, STATE8, true, kOptAhead>(a, s, t, first + i + wave * kOptQuant, kStep, kOptQuant, lane);
        return;
    }
    const long long end = t.n - first < kOptChunk ? t.n : first + kOptChunk;
    for (long long at = first + wave * kOptQuant; at < end; at += kStep) {
        const int left = end - at < kOptQuant ? (int)(end - at) : kOptQuant;
        if (t.wide && left == kOptQuant)
            adamw_256<PARAM, GBF16, STATE8, true, 1>(a, s, t, at, 0, left, lane);
        else
            adamw_256<PARAM, GBF16, STATE8, false, 1>(a, s, t, at, 0, left, lane);
    }
}

// Bound by memory: 30 bytes a value with fp32 moments, a master copy and an fp32 gradient, 18 with 8-bit moments.  778 million
// of the former take 4.18 ms (5.6 TB/s), 123 million of the latter with gradients in bf16 (16 bytes) 338 us (5.8 TB/s).
static __global__ void __launch_bounds__(kOptBlock) adamw_step_k(AdamW a)
{
    const OptChunk c = a.chunks[blockIdx.x];
    const OptTensor t = a.tensors[c.tensor];
    AdamWStep s;
    s.coef = a.clip ? a.clip[1] : 1.f;
    const double lr = a.lr_at ? (double)*a.lr_at : a.lr;
    s.decay = (float)(1.0 - lr * t.weight_decay);
    double bias1 = a.bias1;
    s.inv_root = a.inv_root;
    if (a.step_at) {
        const double step = (double)*a.step_at;
        bias1 = -expm1(step * a.log_beta1);
        s.inv_root = (float)(1.0 / sqrt(-expm1(step * a.log_beta2)));
    }
    s.step_size = (float)(lr / bias1);
    const long long first = (long long)c.chunk * kOptChunk;
    switch ((t.state8 << 2) | (t.grad_bf16 << 1) | t.param_bf16) {
#define GRPO_ADAMW_CASE(S8, GB)                                                                    \
    case (S8 << 2) | (GB << 1):                                                                    \
        adamw_chunk<kParamF32, GB != 0, S8 != 0>(a, s, t, first);                                  \
        break;                                                                                     \
    case (S8 << 2) | (GB << 1) | 1:                                                                \
        if (t.master)                                                                              \
            adamw_chunk<kParamMaster, GB != 0, S8 != 0>(a, s, t, first);                           \
        else                                                                                       \
            adamw_chunk<kParamBf16, GB != 0, S8 != 0>(a, s, t, first);                             \
        break;
        GRPO_ADAMW_CASE(0, 0)
        GRPO_ADAMW_CASE(0, 1)
        GRPO_ADAMW_CASE(1, 0)
        GRPO_ADAMW_CASE(1, 1)
#undef GRPO_ADAMW_CASE
    }
}

// Bound by memory: 778 million gradients in fp32, read once, take 457 us (6.8 TB/s).  14 million, which the caches may hold, take 12, of
// them 4 the second kernel, which adds the workgroups' sums up.
// Squares are exact in fp64 and summed there, each workgroup's chunks in the table's order and the workgroups' sums in theirs:
// the same gradients always give the same norm.
template <bool GBF16, bool WIDE>
__device__ __forceinline__ void load4_grad(const OptTensor &t, long long at, int lane, int left, float (&g)[4])
{
    if constexpr (GBF16)
        load4_bf16<WIDE>((const unsigned short *)t.grad + at, lane, left, g);
    else
        load4_f32<WIDE>((const float *)t.grad + at, lane, left, g);
}
template <bool GBF16>
__device__ __forceinline__ double norm_chunk(const OptTensor &t, long long first)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int kStep = kOptBlock / 64 * kOptQuant, U = kOptChunk / kStep;
    double sum = 0.0;
    if (t.wide && t.n - first >= kOptChunk) {
        float g[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u) load4_grad<GBF16, true>(t, first + u * kStep + wave * kOptQuant, lane, kOptQuant, g[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) sum += (double)g[u][j] * (double)g[u][j];
        return sum;
    }
    const long long end = t.n - first < kOptChunk ? t.n : first + kOptChunk;
    for (long long at = first + wave * kOptQuant; at < end; at += kStep) {
        const int left = end - at < kOptQuant ? (int)(end - at) : kOptQuant;
        float g[4];
        if (t.wide && left == kOptQuant)
            load4_grad<GBF16, true>(t, at, lane, left, g);
        else
            load4_grad<GBF16, false>(t, at, lane, left, g);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += (double)g[j] * (double)g[j];
    }
    return sum;
}

template <int BLOCK>
__device__ __forceinline__ double block_sum_f64(double v, double *lds)  // to all lanes
{
    v = wave_sum_dpp(v);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < BLOCK / 64; ++i) s += lds[i];
    return s;
}

static __global__ void __launch_bounds__(kOptBlock) grad_norm_k(const OptTensor *tensors, const OptChunk *chunks, long long n_chunks, double *partial)
{
    __shared__ double lds[kOptBlock / 64];
    double sum = 0.0;
    for (long long i = blockIdx.x; i < n_chunks; i += gridDim.x) {
        const OptChunk c = chunks[i];
        const OptTensor t = tensors[c.tensor];
        const long long first = (long long)c.chunk * kOptChunk;
        sum += t.grad_bf16 ? norm_chunk<true>(t, first) : norm_chunk<false>(t, first);
    }
    sum = block_sum_f64<kOptBlock>(sum, lds);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

static __global__ void __launch_bounds__(kNormBlocks / 2) grad_norm_total(const double *partial, int n, double max_norm, float *out)
{
    constexpr int BLOCK = kNormBlocks / 2;
    __shared__ double lds[BLOCK / 64];
    const int i = threadIdx.x;
    const double a = i < n ? partial[i] : 0.0, b = i + BLOCK < n ? partial[i + BLOCK] : 0.0;
    const double norm = sqrt(block_sum_f64<BLOCK>(a + b, lds));
    if (threadIdx.x == 0) {
        out[0] = (float)norm;
        out[1] = (float)(!(max_norm > 0.0) || norm <= max_norm ? 1.0 : max_norm / norm);
    }
}

}  // namespace grpo_impl

extern "C" {

size_t grpo_optim_plan_bytes(const grpo_optim_tensor *tensors, int64_t n_tensors)
{
    if (n_tensors < 0 || n_tensors > 0x7fffffffll || (n_tensors > 0 && !tensors)) return 0;
    size_t chunks = 0;
    for (int64_t i = 0; i < n_tensors; ++i) {
        if (tensors[i].n < 0 || tensors[i].n > kOptMaxValues) return 0;
        chunks += (size_t)((tensors[i].n + kOptChunk - 1) / kOptChunk);
    }
    if (chunks > (size_t)kMaxWorkgroups) return 0;
    return align_up(opt_chunks_at(n_tensors) + chunks * sizeof(OptChunk) + 1, 256);
}

grpo_status grpo_optim_plan_build(const grpo_optim_tensor *tensors, int64_t n_tensors, void *table_out, size_t table_bytes,
                                  grpo_optim_plan *plan_out)
{
    if (n_tensors < 0 || n_tensors > 0x7fffffffll) return GRPO_ERR_SHAPE;
    if (!plan_out || !table_out || (n_tensors > 0 && !tensors)) return GRPO_ERR_NULL;
    struct Span {
        uintptr_t from, to;
        bool written;
    };
    std::unique_ptr<Span[]> spans(new (std::nothrow) Span[(size_t)n_tensors * 7 + 1]);
    if (!spans) return GRPO_ERR_WORKSPACE;
    size_t n_spans = 0;
    bool params = true;
    for (int64_t i = 0; i < n_tensors; ++i) {
        const grpo_optim_tensor &t = tensors[i];
        const int pd = raw_enum(t.param_dtype), gd = raw_enum(t.grad_dtype);
        if ((pd != GRPO_F32 && pd != GRPO_BF16) || (gd != GRPO_F32 && gd != GRPO_BF16)) return GRPO_ERR_DTYPE;
        if (t.state_bits != 32 && t.state_bits != 8) return GRPO_ERR_DTYPE;
        if (t.n < 0 || t.n > kOptMaxValues) return GRPO_ERR_SHAPE;
        if (!std::isfinite(t.weight_decay)) return GRPO_ERR_PARAM;
        if (t.n == 0) continue;
        if (!t.param) params = false;
        if (!t.grad) return GRPO_ERR_NULL;
        const size_t n = (size_t)t.n, ps = pd == GRPO_F32 ? 4 : 2, gs = gd == GRPO_F32 ? 4 : 2, ss = t.state_bits / 8;
        if ((uintptr_t)t.grad % gs) return GRPO_ERR_ALIGN;
        spans[n_spans++] = {(uintptr_t)t.grad, (uintptr_t)t.grad + n * gs, false};
        if (!t.param) {
            if (t.master || t.exp_avg || t.exp_avg_sq || t.exp_avg_scale || t.exp_avg_sq_scale) return GRPO_ERR_NULL;
            continue;
        }
        if (!t.exp_avg || !t.exp_avg_sq) return GRPO_ERR_NULL;
        if ((t.state_bits == 8) != (t.exp_avg_scale != nullptr) || (t.state_bits == 8) != (t.exp_avg_sq_scale != nullptr)) return GRPO_ERR_NULL;
        if (t.master && pd != GRPO_BF16) return GRPO_ERR_DTYPE;
        if ((uintptr_t)t.param % ps || (uintptr_t)t.master % 4 || (uintptr_t)t.exp_avg % ss || (uintptr_t)t.exp_avg_sq % ss ||
            (uintptr_t)t.exp_avg_scale % 4 || (uintptr_t)t.exp_avg_sq_scale % 4)
            return GRPO_ERR_ALIGN;
        spans[n_spans++] = {(uintptr_t)t.param, (uintptr_t)t.param + n * ps, true};
        spans[n_spans++] = {(uintptr_t)t.exp_avg, (uintptr_t)t.exp_avg + n * ss, true};
        spans[n_spans++] = {(uintptr_t)t.exp_avg_sq, (uintptr_t)t.exp_avg_sq + n * ss, true};
        if (t.master) spans[n_spans++] = {(uintptr_t)t.master, (uintptr_t)t.master + n * 4, true};
        if (t.state_bits == 8) {
            const size_t blocks = (n + kOptQuant - 1) / kOptQuant;
            spans[n_spans++] = {(uintptr_t)t.exp_avg_scale, (uintptr_t)t.exp_avg_scale + blocks * 4, true};
            spans[n_spans++] = {(uintptr_t)t.exp_avg_sq_scale, (uintptr_t)t.exp_avg_sq_scale + blocks * 4, true};
        }
    }
    const size_t need = grpo_optim_plan_bytes(tensors, n_tensors);
    if (need == 0) return GRPO_ERR_SHAPE;
    if (table_bytes < need) return GRPO_ERR_WORKSPACE;
    // what is written is written by one workgroup and read by nobody else: no array may share a byte with another
    std::sort(spans.get(), spans.get() + n_spans, [](const Span &a, const Span &b) { return a.from < b.from; });
    uintptr_t read_to = 0, written_to = 0;
    for (size_t i = 0; i < n_spans; ++i) {
        if (spans[i].from < written_to || (spans[i].written && spans[i].from < read_to)) return GRPO_ERR_OVERLAP;
        uintptr_t &to = spans[i].written ? written_to : read_to;
        if (spans[i].to > to) to = spans[i].to;
    }
    memset(table_out, 0, need);
    OptChunk *chunk = (OptChunk *)((char *)table_out + opt_chunks_at(n_tensors));
    int64_t n_chunks = 0;
    for (int64_t i = 0; i < n_tensors; ++i) {
        const grpo_optim_tensor &t = tensors[i];
        OptTensor e = {};
        e.param = t.param;
        e.master = t.master;
        e.grad = t.grad;
        e.m = t.exp_avg;
        e.v = t.exp_avg_sq;
        e.m_scale = t.exp_avg_scale;
        e.v_scale = t.exp_avg_sq_scale;
        e.n = t.n;
        e.weight_decay = t.weight_decay;
        e.param_bf16 = raw_enum(t.param_dtype) == GRPO_BF16;
        e.grad_bf16 = raw_enum(t.grad_dtype) == GRPO_BF16;
        e.state8 = t.state_bits == 8;
        const uintptr_t state = (uintptr_t)t.exp_avg | (uintptr_t)t.exp_avg_sq;
        e.wide = (uintptr_t)t.param % (e.param_bf16 ? 8 : 16) == 0 && (uintptr_t)t.master % 16 == 0 &&
                 (uintptr_t)t.grad % (e.grad_bf16 ? 8 : 16) == 0 && state % (e.state8 ? 4 : 16) == 0;
        memcpy((char *)table_out + (size_t)i * sizeof e, &e, sizeof e);
        for (int64_t c = 0; c * kOptChunk < t.n; ++c) chunk[n_chunks++] = {(int)i, (int)c};
    }
    *plan_out = {n_tensors, n_chunks, params ? 1 : 0, 0};
    return GRPO_OK;
}

static grpo_status check_plan(const grpo_optim_plan *plan, const void *table)
{
    if (!plan) return GRPO_ERR_NULL;
    if (plan->n_tensors < 0 || plan->n_chunks < 0 || plan->n_chunks > kMaxWorkgroups) return GRPO_ERR_SHAPE;
    if (plan->n_chunks > 0 && !table) return GRPO_ERR_NULL;
    if ((uintptr_t)table & 255u) return GRPO_ERR_ALIGN;
    return GRPO_OK;
}

size_t grpo_grad_norm_workspace_bytes(void) { return (size_t)kNormBlocks * sizeof(double); }

grpo_status grpo_grad_norm(const grpo_optim_plan *plan, const void *table, double max_norm, float *norm_out, void *workspace,
                           size_t workspace_bytes, void *stream)
{
    const grpo_status bad = check_plan(plan, table);
    if (bad != GRPO_OK) return bad;
    if (std::isnan(max_norm)) return GRPO_ERR_PARAM;
    if (!norm_out) return GRPO_ERR_NULL;
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < grpo_grad_norm_workspace_bytes()) return GRPO_ERR_WORKSPACE;
    // as many chunks to each workgroup
    const int64_t each = (plan->n_chunks + kNormBlocks - 1) / kNormBlocks;
    const int blocks = each > 0 ? (int)((plan->n_chunks + each - 1) / each) : 0;
    const OptTensor *tensors = (const OptTensor *)table;
    const OptChunk *chunks = (const OptChunk *)((const char *)table + opt_chunks_at(plan->n_tensors));
    if (blocks > 0)
        hipLaunchKernelGGL(grad_norm_k, dim3((unsigned)blocks), dim3(kOptBlock), 0, (hipStream_t)stream, tensors, chunks,
                           (long long)plan->n_chunks, (double *)workspace);
    hipLaunchKernelGGL(grad_norm_total, dim3(1), dim3(kNormBlocks / 2), 0, (hipStream_t)stream, (const double *)workspace, blocks, max_norm, norm_out);
    return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}

grpo_status grpo_adamw_step(const grpo_optim_plan *plan, const void *table, int64_t step, const int64_t *step_device, double lr,
                            const float *lr_device, double beta1, double beta2, double eps, const float *clip, void *stream)
{
    const grpo_status bad = check_plan(plan, table);
    if (bad != GRPO_OK) return bad;
    if (plan->n_chunks > 0 && !plan->has_params) return GRPO_ERR_NULL;
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !std::isfinite(eps)) return GRPO_ERR_PARAM;
    if ((!step_device && step < 1) || (!lr_device && !std::isfinite(lr))) return GRPO_ERR_PARAM;
    if (plan->n_chunks == 0) return GRPO_OK;
    AdamW a = {};
    a.tensors = (const OptTensor *)table;
    a.chunks = (const OptChunk *)((const char *)table + opt_chunks_at(plan->n_tensors));
    a.clip = clip;
    a.lr_at = lr_device;
    a.step_at = (const long long *)step_device;
    a.lr = lr;
    a.log_beta1 = std::log(beta1);
    a.log_beta2 = std::log(beta2);
    a.beta1 = (float)beta1;
    a.one_beta1 = (float)(1.0 - beta1);
    a.beta2 = (float)beta2;
    a.one_beta2 = (float)(1.0 - beta2);
    a.eps = (float)eps;
    if (!step_device) {
        a.bias1 = 1.0 - std::pow(beta1, (double)step);
        a.inv_root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    }
    hipLaunchKernelGGL(adamw_step_k, dim3((unsigned)plan->n_chunks), dim3(kOptBlock), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}

}  // extern "C"
