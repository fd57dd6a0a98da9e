// The norms around a block of the model, with the block's gate and the scale it is added to the residual stream with, and
// their gradients.  Part of grpo.hip's translation unit.
//
//   x' = x + s g (.) f r1 (.) w1      r1 = 1 / sqrt(mean(f^2) + eps)      f: the block's output, x: the residual stream
//   h  = x' r2 (.) w2                 r2 = 1 / sqrt(mean(x'^2) + eps)     h: what the next block, or the head, takes
//
// and with y2 = x' r2, a = w2 (.) dh, y1 = f r1:
//
//   dx  = D = dx' + r2 (a - y2 mean(a (.) y2))          dw2 = sum over rows of dh (.) y2
//   t   = s g (.) w1 (.) D                              dw1 = sum over rows of s g (.) D (.) y1
//   df  = r1 (t - y1 mean(t (.) y1))                    dg  = s w1 (.) D (.) y1 (summed over rows where one gate serves all)
//
// Both norms' 1/sqrt are formed again in the backward: their sums go along with those it needs anyway.
//
// Bound by memory.  Rows stay in registers between the passes over them, so that they are read once: 16384 x 5120 with a residual in fp32,
// the rest in bf16 and a gate for every row take 190 us forward (14 bytes a value, 6.2 TB/s) and 345 backward (22 bytes,
// 5.3 TB/s), where kernels that read a row again for every pass took 322 and 1028.  The backward holds 12 registers for each of a
// lane's values, which leaves two wavefronts to a SIMD: with sums over rows in LDS instead (10 registers) it was no faster
// (394 us), with the next row asked for in front of the last pass neither (360).

namespace __attribute__((visibility("hidden"))) grpo_impl {

struct BlockNorm {
    const char *x, *f, *w1, *g, *w2, *dh, *dxo;  // forward: x = the residual stream; backward: x = x'
    char *xo, *h;                                // forward
    char *dx, *df, *dg;                          // backward; dg here where every row has a gate
    float *part;                                 // backward: [grid][2][d] sums over a workgroup's rows
    long long xs, fs, gs, dhs, dxos, xos, hs, dxs, dfs, dgs;  // row pitches in bytes
    long long n;
    int d;
    float scale, eps, inv_d;
};

// VEC neighbours of a row as they lie in memory: 16 bytes, or 8 of bf16 beside 16 of fp32.
template <grpo_dtype DT, int VEC>
struct RawVec {
    static_assert(VEC == Elem<DT>::EPV, "16 bytes");
    u32x4 v;
    __device__ __forceinline__ void get(float (&f)[VEC]) const { unpack<DT>(v, f); }
    __device__ __forceinline__ void set(const float (&f)[VEC]) { v = pack<DT>(f); }
};
template <>
struct RawVec<GRPO_BF16, 4> {
    u32x2 v;
    __device__ __forceinline__ void get(float (&f)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f[2 * i] = as_f32(v[i] << 16);
            f[2 * i + 1] = as_f32(v[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&f)[4]) { v = u32x2{bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3])}; }
};

// The neighbours from column col on.  RAGGED: the row may end inside them; zeros behind its end.  ONCE: nobody reads them again.
template <grpo_dtype DT, int VEC, bool RAGGED = true, bool ONCE = true>
__device__ __forceinline__ RawVec<DT, VEC> raw_load(const char *row, int col, int d)
{
    RawVec<DT, VEC> r;
    if (!RAGGED || col + VEC <= d) {
        typedef decltype(r.v) V;
        const V *at = (const V *)(row + (size_t)col * Elem<DT>::BYTES);
        r.v = ONCE ? __builtin_nontemporal_load(at) : *at;
    } else {
        float f[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] = col + i < d ? load_elem<DT>(row, col + i) : 0.f;
        r.set(f);
    }
    return r;
}
template <grpo_dtype DT, int VEC, bool RAGGED = true>
__device__ __forceinline__ void row_load(const char *row, int col, int d, float (&v)[VEC])
{
    raw_load<DT, VEC, RAGGED, false>(row, col, d).get(v);  // weights, and rows that are read again
}
template <grpo_dtype DT, int VEC, bool RAGGED = true>
__device__ __forceinline__ void row_store(char *row, int col, int d, const float (&v)[VEC])
{
    RawVec<DT, VEC> r;
    if (!RAGGED || col + VEC <= d) {
        typedef decltype(r.v) V;
        r.set(v);
        __builtin_nontemporal_store(r.v, (V *)(row + (size_t)col * Elem<DT>::BYTES));
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (col + i < d) store_elem<DT>(row, col + i, v[i]);
    }
}

constexpr int kNormBlock = 256, kWideBlock = 1024;
constexpr int kWideSums = 19456;  // columns whose two sums fit the LDS of a CU, beside the reductions
constexpr long long kNormFwdGrid = 65536;
constexpr long long kNormGrid = 1024;  // workgroups of the backward at most, each with a row of partial sums

// The sum over the TPR lanes that share a row, to all of them: a wavefront, or the workgroup (lds: a place for each wavefront that
// nobody reads any more).
template <int TPR>
__device__ __forceinline__ float row_sum_of(float v, float *lds)
{
    if constexpr (TPR == 64)
        return wave_sum(v);
    else
        return block_sum<TPR>(v, lds);
}

// Where a lane loads from: at column 0 if the row has none for it, and blank() takes out what would go into a sum.  Nothing is under
// a condition but the stores: what is loaded under one is waited for where it ends, weights of every vector one after the other.
// (Where rows end inside a vector its loads are.  To patch that vector in behind loads without conditions takes longer: 8192 x
// 5121 bf16 forward 125 us and 139, backward with an fp32 residual 275 and 335.)
template <bool RAGGED>
__device__ __forceinline__ int held_column(int col, int d)
{
    return RAGGED || col < d ? col : 0;
}
template <grpo_dtype DT, int VEC>
__device__ __forceinline__ void blank(RawVec<DT, VEC> &r, bool there)
{
#pragma unroll
    for (int i = 0; i < (int)(sizeof(r.v) / 4); ++i) r.v[i] = there ? r.v[i] : 0u;
}

// The weights of a lane's columns, once for all of its rows.
template <grpo_dtype DT, int VEC, int TPR, int NV, bool RAGGED>
__device__ __forceinline__ void load_weights(const BlockNorm &p, int t, RawVec<DT, VEC> (&w1)[NV], RawVec<DT, VEC> (&w2)[NV])
{
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int col = held_column<RAGGED>((i * TPR + t) * VEC, p.d);
        if (p.w1) w1[i] = raw_load<DT, VEC, RAGGED, false>(p.w1, col, p.d);
        if (p.w2) w2[i] = raw_load<DT, VEC, RAGGED, false>(p.w2, col, p.d);
    }
}

// Rows that stay in registers between the passes over them: TPR lanes to a row, NV vectors to a lane.
template <grpo_dtype RT, grpo_dtype DT, int TPR, int NV, bool RAGGED>
__global__ void __launch_bounds__(TPR < kNormBlock ? kNormBlock : TPR) block_norm_fwd_held(BlockNorm p)
{
    constexpr int VEC = Elem<RT>::EPV, BLOCK = TPR < kNormBlock ? kNormBlock : TPR, ROWS = BLOCK / TPR;
    __shared__ float lds[2][2][BLOCK / 64];
    const int t = threadIdx.x % TPR;
    RawVec<DT, VEC> w1r[NV], w2r[NV];
    load_weights<DT, VEC, TPR, NV, RAGGED>(p, t, w1r, w2r);
    int turn = 0;
    for (long long row = (long long)blockIdx.x * ROWS + threadIdx.x / TPR; row < p.n; row += (long long)gridDim.x * ROWS, turn ^= 1) {
        const char *x = p.x + row * p.xs, *f = p.f ? p.f + row * p.fs : nullptr, *g = p.g ? p.g + row * p.gs : nullptr;
        RawVec<RT, VEC> xr[NV];
        RawVec<DT, VEC> fr[NV], gr[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = held_column<RAGGED>((i * TPR + t) * VEC, p.d);
            if (f) fr[i] = raw_load<DT, VEC, RAGGED>(f, col, p.d);
            xr[i] = raw_load<RT, VEC, RAGGED>(x, col, p.d);
            if (g) gr[i] = raw_load<DT, VEC, RAGGED>(g, col, p.d);
        }
        float r1 = p.scale;
        if (p.w1) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                blank(fr[i], (i * TPR + t) * VEC < p.d);
                float b[VEC];
                fr[i].get(b);
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum += b[e] * b[e];
            }
            r1 *= 1.f / sqrtf(row_sum_of<TPR>(sum, lds[turn][0]) * p.inv_d + p.eps);
        }
        float sum = 0.f;
        float v[NV][VEC];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool there = (i * TPR + t) * VEC < p.d;
            const int col = (i * TPR + t) * VEC;
            xr[i].get(v[i]);
            if (f) {
                float b[VEC], w[VEC];
                fr[i].get(b);
                if (p.w1) {
                    w1r[i].get(w);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) b[e] *= w[e];
                }
                if (g) {
                    gr[i].get(w);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) b[e] *= w[e];
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[i][e] += r1 * b[e];
                if (there) row_store<RT, VEC, RAGGED>(p.xo + row * p.xos, col, p.d, v[i]);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum += there ? v[i][e] * v[i][e] : 0.f;
        }
        if (!p.w2) continue;
        const float r2 = 1.f / sqrtf(row_sum_of<TPR>(sum, lds[turn][1]) * p.inv_d + p.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool there = (i * TPR + t) * VEC < p.d;
            const int col = (i * TPR + t) * VEC;
            float w[VEC];
            w2r[i].get(w);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[i][e] *= r2 * w[e];
            if (there) row_store<DT, VEC, RAGGED>(p.h + row * p.hs, col, p.d, v[i]);
        }
    }
}

// What is added to the residual stream, without the scale: the block's output, normed, weighted and gated.
template <grpo_dtype DT, int VEC>
__device__ __forceinline__ void branch(const BlockNorm &p, const char *g, int col, float r1, float (&f)[VEC])
{
    float w[VEC];
    if (p.w1) {
        row_load<DT, VEC>(p.w1, col, p.d, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] *= r1 * w[i];
    }
    if (g) {
        row_load<DT, VEC>(g, col, p.d, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] *= w[i];
    }
}

// Rows that are too wide to hold: read again for every pass.
template <grpo_dtype RT, grpo_dtype DT>
__global__ void __launch_bounds__(kNormBlock) block_norm_fwd_streamed(BlockNorm p)
{
    constexpr int VEC = 16 / Elem<RT>::BYTES;
    __shared__ float lds[2][kNormBlock / 64];
    for (long long row = blockIdx.x; row < p.n; row += gridDim.x) {
        const char *x = p.x + row * p.xs, *f = p.f ? p.f + row * p.fs : nullptr, *g = p.g ? p.g + row * p.gs : nullptr;
        float r1 = 1.f, r2 = 0.f, sum = 0.f;
        if (p.w1) {
            for (int col = threadIdx.x * VEC; col < p.d; col += kNormBlock * VEC) {
                float v[VEC];
                row_load<DT, VEC>(f, col, p.d, v);
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum += v[i] * v[i];
            }
            r1 = 1.f / sqrtf(block_sum<kNormBlock>(sum, lds[0]) * p.inv_d + p.eps);
        }
        sum = 0.f;
        for (int pass = p.w2 ? 0 : 1; pass < 2; ++pass) {
            for (int col = threadIdx.x * VEC; col < p.d; col += kNormBlock * VEC) {
                float v[VEC], b[VEC];
                row_load<RT, VEC>(x, col, p.d, v);
                if (f) {
                    row_load<DT, VEC>(f, col, p.d, b);
                    branch<DT, VEC>(p, g, col, r1, b);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) v[i] += p.scale * b[i];
                }
                if (pass == 0) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) sum += v[i] * v[i];
                    continue;
                }
                if (f) row_store<RT, VEC>(p.xo + row * p.xos, col, p.d, v);
                if (p.w2) {
                    row_load<DT, VEC>(p.w2, col, p.d, b);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) v[i] *= r2 * b[i];
                    row_store<DT, VEC>(p.h + row * p.hs, col, p.d, v);
                }
            }
            if (pass == 0) r2 = 1.f / sqrtf(block_sum<kNormBlock>(sum, lds[1]) * p.inv_d + p.eps);
        }
        __syncthreads();  // the next row's sums go where this one's were
    }
}

// Three sums behind one barrier.
template <int TPR>
__device__ __forceinline__ void row_sum3_of(float &a, float &b, float &c, float (*lds)[4])
{
    a = wave_sum(a);
    b = wave_sum(b);
    c = wave_sum(c);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) {
            float *at = lds[threadIdx.x >> 6];
            at[0] = a;
            at[1] = b;
            at[2] = c;
        }
        lds_barrier();
        a = lds[0][0];
        b = lds[0][1];
        c = lds[0][2];
#pragma unroll
        for (int w = 1; w < TPR / 64; ++w) {
            a += lds[w][0];
            b += lds[w][1];
            c += lds[w][2];
        }
    }
}

// Rows that stay in registers, and with them the sums over the workgroup's rows.
template <grpo_dtype RT, grpo_dtype DT, int TPR, int NV, bool RAGGED>
__global__ void __launch_bounds__(TPR < kNormBlock ? kNormBlock : TPR, 2) block_norm_bwd_held(BlockNorm p)
{
    constexpr int VEC = Elem<RT>::EPV, BLOCK = TPR < kNormBlock ? kNormBlock : TPR, ROWS = BLOCK / TPR;
    __shared__ float lds[2][BLOCK / 64][4], lds_t[2][BLOCK / 64];
    const int t = threadIdx.x % TPR;
    float acc2[NV][VEC] = {}, acc1[NV][VEC] = {};
    RawVec<RT, VEC> xr[NV], dr[NV];
    RawVec<DT, VEC> hr[NV], fr[NV], gr[NV], w1r[NV], w2r[NV];
    load_weights<DT, VEC, TPR, NV, RAGGED>(p, t, w1r, w2r);
    const long long step = (long long)gridDim.x * ROWS;
    long long row = (long long)blockIdx.x * ROWS + threadIdx.x / TPR;
    for (int turn = 0; row < p.n; row += step, turn ^= 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = held_column<RAGGED>((i * TPR + t) * VEC, p.d);
            if (p.w2) {
                xr[i] = raw_load<RT, VEC, RAGGED>(p.x + row * p.xs, col, p.d);
                hr[i] = raw_load<DT, VEC, RAGGED>(p.dh + row * p.dhs, col, p.d);
            }
            if (p.f) fr[i] = raw_load<DT, VEC, RAGGED>(p.f + row * p.fs, col, p.d);
            if (p.dxo) dr[i] = raw_load<RT, VEC, RAGGED>(p.dxo + row * p.dxos, col, p.d);
            if (p.g) gr[i] = raw_load<DT, VEC, RAGGED>(p.g + row * p.gs, col, p.d);
        }
        float sx = 0.f, sax = 0.f, sf = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool there = (i * TPR + t) * VEC < p.d;
            float u[VEC], v[VEC], w[VEC];
            if (p.w2) {
                blank(xr[i], there);
                xr[i].get(v);
                hr[i].get(u);
                w2r[i].get(w);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    sx += v[e] * v[e];
                    sax += u[e] * w[e] * v[e];
                }
            }
            if (p.w1) {
                blank(fr[i], there);
                fr[i].get(v);
#pragma unroll
                for (int e = 0; e < VEC; ++e) sf += v[e] * v[e];
            }
        }
        row_sum3_of<TPR>(sx, sax, sf, lds[turn]);
        const float r2 = p.w2 ? 1.f / sqrtf(sx * p.inv_d + p.eps) : 0.f;
        const float c2 = sax * r2 * p.inv_d;  // mean(a y2)
        const float r1 = p.w1 ? 1.f / sqrtf(sf * p.inv_d + p.eps) : 1.f;
        float D[NV][VEC];
        float sty = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool there = (i * TPR + t) * VEC < p.d;
            const int col = (i * TPR + t) * VEC;
            float u[VEC], v[VEC], w[VEC];
            if (p.dxo) {
                dr[i].get(D[i]);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) D[i][e] = 0.f;
            }
            if (p.w2) {
                xr[i].get(v);
                hr[i].get(u);
                w2r[i].get(w);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float y2 = v[e] * r2;
                    D[i][e] += r2 * (u[e] * w[e] - y2 * c2);
                    acc2[i][e] += u[e] * y2;
                }
            }
            if (there) row_store<RT, VEC, RAGGED>(p.dx + row * p.dxs, col, p.d, D[i]);
            if (!p.f) continue;
            // from here on D is s D, and with a weight and a gate t
            fr[i].get(v);
            float sy[VEC];  // s D y1
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                v[e] *= r1;
                D[i][e] *= p.scale;
                sy[e] = D[i][e] * v[e];
            }
            if (p.w1) {
                w1r[i].get(w);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) w[e] = 1.f;
            }
            if (p.g) {
                gr[i].get(u);
                if (p.dg) {
                    float dg[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) dg[e] = sy[e] * w[e];
                    if (there) row_store<DT, VEC, RAGGED>(p.dg + row * p.dgs, col, p.d, dg);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sy[e] *= u[e];
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) w[e] *= u[e];
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                acc1[i][e] += sy[e];
                D[i][e] *= w[e];
                sty += D[i][e] * v[e];
            }
        }
        if (p.f) {
            float c1 = 0.f;
            if (p.w1) c1 = row_sum_of<TPR>(sty, lds_t[turn]) * p.inv_d * r1;  // mean(t y1) r1
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int col = (i * TPR + t) * VEC;
                if (p.w1) {
                    float v[VEC];
                    fr[i].get(v);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) D[i][e] = r1 * (D[i][e] - v[e] * c1);
                }
                if (col < p.d) row_store<DT, VEC, RAGGED>(p.df + row * p.dfs, col, p.d, D[i]);
            }
        }
    }
    // one row of sums to a workgroup
    float *part = p.part + (size_t)blockIdx.x * 2 * p.d;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (i * TPR + t) * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (col + e < p.d) {
                    part[col + e] = acc2[i][e];
                    part[p.d + col + e] = acc1[i][e];
                }
        }
    } else {
        __shared__ float sums[TPR * NV * VEC];
        for (int which = 0; which < 2; ++which) {
            for (int r = 0; r < ROWS; ++r) {
                if (threadIdx.x / TPR == r) {
#pragma unroll
                    for (int i = 0; i < NV; ++i)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            float &s = sums[(i * TPR + t) * VEC + e];
                            s = (r ? s : 0.f) + (which ? acc1[i][e] : acc2[i][e]);
                        }
                }
                __syncthreads();
            }
            for (int col = threadIdx.x; col < p.d; col += BLOCK) part[(size_t)which * p.d + col] = sums[col];
            __syncthreads();
        }
    }
}

// Wider rows: read again for every pass, each lane's columns the same in all.  The sums over rows are in LDS where they fit (SUMS_LDS),
// else in the workspace: 4096 x 16384 bf16 358 us
// and 794, with an fp32 residual 479 and 836.
template <grpo_dtype RT, grpo_dtype DT, bool SUMS_LDS>
__global__ void __launch_bounds__(kWideBlock) block_norm_bwd_streamed(BlockNorm p)
{
    extern __shared__ __align__(16) float wide_sums[];
    constexpr int VEC = 16 / Elem<RT>::BYTES;
    __shared__ float lds[4][kWideBlock / 64];
    float *part = p.part + (size_t)blockIdx.x * 2 * p.d, *sums = SUMS_LDS ? wide_sums : part;
    for (long long row = blockIdx.x; row < p.n; row += gridDim.x) {
        const char *x = p.x + row * p.xs, *f = p.f ? p.f + row * p.fs : nullptr, *g = p.g ? p.g + row * p.gs : nullptr;
        const char *dh = p.w2 ? p.dh + row * p.dhs : nullptr, *dxo = p.dxo ? p.dxo + row * p.dxos : nullptr;
        float sx = 0.f, sax = 0.f, sf = 0.f;
        for (int col = threadIdx.x * VEC; col < p.d; col += kWideBlock * VEC) {
            float v[VEC], w[VEC], u[VEC];
            if (p.w2) {
                row_load<RT, VEC>(x, col, p.d, v);
                row_load<DT, VEC>(dh, col, p.d, u);
                row_load<DT, VEC>(p.w2, col, p.d, w);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    sx += v[i] * v[i];
                    sax += u[i] * w[i] * v[i];
                }
            }
            if (p.w1) {
                row_load<DT, VEC>(f, col, p.d, v);
#pragma unroll
                for (int i = 0; i < VEC; ++i) sf += v[i] * v[i];
            }
        }
        block_sum2<kWideBlock>(sx, sax, lds[0], lds[1]);
        const float r1 = p.w1 ? 1.f / sqrtf(block_sum<kWideBlock>(sf, lds[2]) * p.inv_d + p.eps) : 1.f;
        const float r2 = 1.f / sqrtf(sx * p.inv_d + p.eps);
        const float c2 = sax * r2 * p.inv_d;  // mean(a y2)
        float sty = 0.f, c1 = 0.f;
        for (int pass = p.w1 ? 0 : 1; pass < 2; ++pass) {
            for (int col = threadIdx.x * VEC; col < p.d; col += kWideBlock * VEC) {
                float v[VEC], w[VEC], u[VEC], D[VEC] = {};
                if (dxo) row_load<RT, VEC>(dxo, col, p.d, D);
                if (p.w2) {
                    row_load<RT, VEC>(x, col, p.d, v);
                    row_load<DT, VEC>(dh, col, p.d, u);
                    row_load<DT, VEC>(p.w2, col, p.d, w);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        const float y2 = v[i] * r2;
                        D[i] += r2 * (u[i] * w[i] - y2 * c2);
                        v[i] = u[i] * y2;  // its share of dw2
                    }
                    if (pass == 1)
#pragma unroll
                        for (int i = 0; i < VEC; ++i)
                            if (col + i < p.d) sums[col + i] = (row == blockIdx.x ? 0.f : sums[col + i]) + v[i];
                }
                if (pass == 1) row_store<RT, VEC>(p.dx + row * p.dxs, col, p.d, D);
                if (!f) continue;
                float y[VEC], gate[VEC], w1[VEC], t[VEC], sum[VEC];
                row_load<DT, VEC>(f, col, p.d, y);
                if (p.w1) row_load<DT, VEC>(p.w1, col, p.d, w1);
                if (g) row_load<DT, VEC>(g, col, p.d, gate);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    y[i] *= r1;
                    if (!p.w1) w1[i] = 1.f;
                    if (!g) gate[i] = 1.f;
                    const float sD = p.scale * D[i];
                    t[i] = sD * gate[i] * w1[i];
                    sum[i] = sD * y[i] * (p.gs ? gate[i] : 1.f);
                    gate[i] = sD * y[i] * w1[i];  // its gradient
                    if (pass == 0) sty += t[i] * y[i];
                }
                if (pass == 0) continue;
                if (p.w1) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) t[i] = r1 * (t[i] - y[i] * c1);
                }
                row_store<DT, VEC>(p.df + row * p.dfs, col, p.d, t);
                if (p.dg) row_store<DT, VEC>(p.dg + row * p.dgs, col, p.d, gate);
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (col + i < p.d) sums[p.d + col + i] = (row == blockIdx.x ? 0.f : sums[p.d + col + i]) + sum[i];
            }
            if (pass == 0) c1 = block_sum<kWideBlock>(sty, lds[3]) * p.inv_d;
        }
        __syncthreads();
    }
    if constexpr (SUMS_LDS)
        for (int i = threadIdx.x; i < 2 * p.d; i += kWideBlock) part[i] = wide_sums[i];
}

// The workgroups' sums, added up in fp64: 64 columns to a workgroup, a sixteenth of the sums to each of its wavefronts, which
// then are added in their order.  With one gate for all rows (or none) the second sum is that of s D (.) y1, which gives both
// dw1, times the gate, and the gate's gradient, times w1.
template <grpo_dtype DT>
__global__ void __launch_bounds__(1024) block_norm_columns(const float *part, int blocks, int d, const char *w1, const char *gate_row,
                                                           float *dw1, float *dgate_row, float *dw2, int accumulate)
{
    __shared__ double lds[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = blockIdx.x * 64 + lane, which = blockIdx.y;
    if (which == 0 ? !dw2 : !dw1 && !dgate_row) return;
    double s = 0.0;
    if (col < d) {
        const float *at = part + (size_t)which * d + col;
#pragma unroll 8
        for (int b = wave; b < blocks; b += 16) s += (double)at[(size_t)b * 2 * d];
    }
    lds[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || col >= d) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += lds[w][lane];
    if (which == 0) {
        dw2[col] = accumulate ? dw2[col] + (float)s : (float)s;
        return;
    }
    if (dw1) {
        const float v = (float)s * (gate_row ? load_elem<DT>(gate_row, col) : 1.f);
        dw1[col] = accumulate ? dw1[col] + v : v;
    }
    if (dgate_row) {
        const float v = (float)s * (w1 ? load_elem<DT>(w1, col) : 1.f);
        dgate_row[col] = accumulate ? dgate_row[col] + v : v;
    }
}

constexpr int64_t kNormMaxWidth = 1 << 20;

// A [n, d] array: present, on 16-byte boundaries, rows at least d apart.
static grpo_status check_rows(const void *p, int64_t stride, int64_t d, int dtype, bool wanted)
{
    if ((p != nullptr) != wanted) return GRPO_ERR_NULL;
    if (!p) return GRPO_OK;
    if (stride < d) return GRPO_ERR_SHAPE;
    const int64_t bytes = dtype == GRPO_BF16 ? 2 : 4;
    if (((uintptr_t)p & 15u) || ((stride * bytes) & 15)) return GRPO_ERR_ALIGN;
    return GRPO_OK;
}

static grpo_status check_block_norm(int rt, int dt, const void *block, const void *w1, const void *gate, int64_t gate_stride, const void *w2,
                                    int64_t n, int64_t d, double scale, double eps)
{
    if ((rt != GRPO_F32 && rt != GRPO_BF16) || (dt != GRPO_F32 && dt != GRPO_BF16) || (rt == GRPO_BF16 && dt == GRPO_F32)) return GRPO_ERR_DTYPE;
    if (n < 0 || d <= 0 || d > kNormMaxWidth || gate_stride < 0) return GRPO_ERR_SHAPE;
    if (!std::isfinite(scale) || !(eps >= 0.0) || !std::isfinite(eps)) return GRPO_ERR_PARAM;
    if (n > 0 && !block && (w1 || gate || !w2)) return GRPO_ERR_NULL;
    if (gate && gate_stride != 0 && gate_stride < d) return GRPO_ERR_SHAPE;
    if (((uintptr_t)w1 | (uintptr_t)w2 | (uintptr_t)gate) & 15u) return GRPO_ERR_ALIGN;
    if (gate && ((gate_stride * (dt == GRPO_BF16 ? 2 : 4)) & 15)) return GRPO_ERR_ALIGN;
    return GRPO_OK;
}

static BlockNorm block_norm_params(int rt, int dt, const void *x, int64_t xs, const void *block, int64_t fs, const void *w1, const void *gate,
                                   int64_t gs, const void *w2, int64_t n, int64_t d, double scale, double eps)
{
    const int64_t rb = rt == GRPO_BF16 ? 2 : 4, db = dt == GRPO_BF16 ? 2 : 4;
    BlockNorm p = {};
    p.x = (const char *)x;
    p.xs = xs * rb;
    p.f = (const char *)block;
    p.fs = fs * db;
    p.w1 = (const char *)w1;
    p.g = (const char *)gate;
    p.gs = gs * db;
    p.w2 = (const char *)w2;
    p.n = n;
    p.d = (int)d;
    p.scale = (float)scale;
    p.eps = (float)eps;
    p.inv_d = (float)(1.0 / (double)d);
    return p;
}

// Which kernel takes rows of d: X(lanes to a row, vectors to a lane) of the list for 8 or 4 values to a vector, the first
// that holds a row, else the streamed one.  A wavefront to a row, several to a workgroup, as far as its registers go; then as many wavefronts as
// leave a lane 20 values backward, 32 forward: with fewer the workgroups of a CU are too few to hide what a row waits for (backward of 5120
// on 640 lanes 399 us, on 320 376, on 256 345), with more its registers run out.
#define GRPO_NORM_FWD_8(X) X(64, 1) X(64, 2) X(256, 1) X(256, 2) X(320, 2) X(256, 4) X(512, 4)
#define GRPO_NORM_FWD_4(X) X(64, 1) X(64, 2) X(64, 4) X(256, 2) X(256, 4) X(256, 5) X(256, 8) X(512, 8)
#define GRPO_NORM_BWD_8(X) X(64, 1) X(64, 2) X(256, 1) X(256, 2) X(320, 2) X(512, 2)
#define GRPO_NORM_BWD_4(X) X(64, 1) X(64, 2) X(64, 4) X(256, 2) X(256, 4) X(256, 5) X(512, 4) X(512, 5)
#define GRPO_NORM_CASE(KERNEL, MOST, TPR, NV)                                                                                        \
    if (p.d <= TPR * NV * Elem<RT>::EPV) {                                                                                           \
        constexpr int BLOCK = TPR < kNormBlock ? kNormBlock : TPR, ROWS = BLOCK / TPR;                                              \
        const long long blocks = (p.n + ROWS - 1) / ROWS, grid = blocks < MOST ? blocks : MOST;                                      \
        if (p.d % Elem<RT>::EPV)                                                                                                     \
            hipLaunchKernelGGL((KERNEL<RT, DT, TPR, NV, true>), dim3((unsigned)grid), dim3(BLOCK), 0, st, p);                        \
        else                                                                                                                         \
            hipLaunchKernelGGL((KERNEL<RT, DT, TPR, NV, false>), dim3((unsigned)grid), dim3(BLOCK), 0, st, p);                       \
        return (int)grid;                                                                                                            \
    }
template <grpo_dtype RT, grpo_dtype DT>
static int launch_block_norm_fwd(const BlockNorm &p, hipStream_t st)
{
#define GRPO_NORM_FWD(TPR, NV) GRPO_NORM_CASE(block_norm_fwd_held, kNormFwdGrid, TPR, NV)
    if constexpr (Elem<RT>::EPV == 8) {
        GRPO_NORM_FWD_8(GRPO_NORM_FWD)
    } else {
        GRPO_NORM_FWD_4(GRPO_NORM_FWD)
    }
#undef GRPO_NORM_FWD
    const long long grid = p.n < kNormFwdGrid ? p.n : kNormFwdGrid;
    hipLaunchKernelGGL((block_norm_fwd_streamed<RT, DT>), dim3((unsigned)grid), dim3(kNormBlock), 0, st, p);
    return (int)grid;
}

template <grpo_dtype RT, grpo_dtype DT>
static int launch_block_norm_bwd_rows(const BlockNorm &p, hipStream_t st)  // workgroups, and rows of partial sums
{
    if (p.n == 0) return 0;
#define GRPO_NORM_BWD(TPR, NV) GRPO_NORM_CASE(block_norm_bwd_held, kNormGrid, TPR, NV)
    if constexpr (Elem<RT>::EPV == 8) {
        GRPO_NORM_BWD_8(GRPO_NORM_BWD)
    } else {
        GRPO_NORM_BWD_4(GRPO_NORM_BWD)
    }
#undef GRPO_NORM_BWD
    const long long cus = cu_count(), grid = p.n < cus ? p.n : cus;
    if (p.d <= kWideSums) {
        const unsigned lds = 2u * (unsigned)p.d * 4u;
        static std::atomic<bool> attr_done[64];  // setting the attribute twice is harmless
        int dev = 0;
        if (hipGetDevice(&dev) == hipSuccess && dev >= 0 && dev < 64 && !attr_done[dev].load()) {
            if (hipFuncSetAttribute((const void *)block_norm_bwd_streamed<RT, DT, true>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                    kWideSums * 8) == hipSuccess)
                attr_done[dev].store(true);
        }
        hipLaunchKernelGGL((block_norm_bwd_streamed<RT, DT, true>), dim3((unsigned)grid), dim3(kWideBlock), lds, st, p);
    } else {
        hipLaunchKernelGGL((block_norm_bwd_streamed<RT, DT, false>), dim3((unsigned)grid), dim3(kWideBlock), 0, st, p);
    }
    return (int)grid;
}

template <grpo_dtype RT, grpo_dtype DT>
static void launch_block_norm_bwd(const BlockNorm &p, hipStream_t st, float *dw1, float *dgate_row, float *dw2, int accumulate)
{
    const int blocks = launch_block_norm_bwd_rows<RT, DT>(p, st);
    if (dw1 || dgate_row || dw2)
        hipLaunchKernelGGL((block_norm_columns<DT>), dim3((unsigned)((p.d + 63) / 64), 2), dim3(1024), 0, st, p.part, blocks, p.d, p.w1,
                           p.gs ? nullptr : p.g, dw1, dgate_row, dw2, accumulate);
}

}  // namespace grpo_impl

extern "C" {

grpo_status grpo_block_norm_fwd(const void *residual, int64_t residual_stride, grpo_dtype residual_dtype, const void *block,
                                int64_t block_stride, const void *post_weight, const void *gate, int64_t gate_stride,
                                const void *pre_weight, grpo_dtype dtype, int64_t n_tokens, int64_t d_model, double residual_scale,
                                double eps, void *residual_out, int64_t residual_out_stride, void *hidden, int64_t hidden_stride, void *stream)
{
    const int rt = raw_enum(residual_dtype), dt = raw_enum(dtype);
    grpo_status bad = check_block_norm(rt, dt, block, post_weight, gate, gate_stride, pre_weight, n_tokens, d_model, residual_scale, eps);
    if (bad != GRPO_OK) return bad;
    if (n_tokens == 0) return GRPO_OK;
    if ((bad = check_rows(residual, residual_stride, d_model, rt, true)) != GRPO_OK) return bad;
    if ((bad = check_rows(block, block_stride, d_model, dt, block != nullptr)) != GRPO_OK) return bad;
    if ((bad = check_rows(residual_out, residual_out_stride, d_model, rt, block != nullptr)) != GRPO_OK) return bad;
    if ((bad = check_rows(hidden, hidden_stride, d_model, dt, pre_weight != nullptr)) != GRPO_OK) return bad;
    BlockNorm p = block_norm_params(rt, dt, residual, residual_stride, block, block_stride, post_weight, gate, gate_stride, pre_weight,
                                    n_tokens, d_model, residual_scale, eps);
    p.xo = (char *)residual_out;
    p.xos = residual_out_stride * (rt == GRPO_BF16 ? 2 : 4);
    p.h = (char *)hidden;
    p.hs = hidden_stride * (dt == GRPO_BF16 ? 2 : 4);
    hipStream_t st = (hipStream_t)stream;
    if (rt == GRPO_BF16)
        launch_block_norm_fwd<GRPO_BF16, GRPO_BF16>(p, st);
    else if (dt == GRPO_BF16)
        launch_block_norm_fwd<GRPO_F32, GRPO_BF16>(p, st);
    else
        launch_block_norm_fwd<GRPO_F32, GRPO_F32>(p, st);
    return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}

size_t grpo_block_norm_workspace_bytes(int64_t n_tokens, int64_t d_model)
{
    if (n_tokens < 0 || d_model <= 0 || d_model > kNormMaxWidth) return 0;
    const size_t blocks = (size_t)(n_tokens < kNormGrid ? n_tokens : kNormGrid);
    return align_up(blocks * 2 * (size_t)d_model * 4 + 1, 256);
}

grpo_status grpo_block_norm_bwd(const void *residual_out, int64_t residual_out_stride, grpo_dtype residual_dtype, const void *block,
                                int64_t block_stride, const void *post_weight, const void *gate, int64_t gate_stride,
                                const void *pre_weight, grpo_dtype dtype, int64_t n_tokens, int64_t d_model, double residual_scale,
                                double eps, const void *grad_hidden, int64_t grad_hidden_stride, const void *grad_residual_out,
                                int64_t grad_residual_out_stride, void *grad_residual, int64_t grad_residual_stride, void *grad_block,
                                int64_t grad_block_stride, void *grad_gate, int64_t grad_gate_stride, float *grad_post_weight,
                                float *grad_pre_weight, int accumulate_grad_weights, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rt = raw_enum(residual_dtype), dt = raw_enum(dtype);
    grpo_status bad = check_block_norm(rt, dt, block, post_weight, gate, gate_stride, pre_weight, n_tokens, d_model, residual_scale, eps);
    if (bad != GRPO_OK) return bad;
    if ((post_weight != nullptr) != (grad_post_weight != nullptr) || (pre_weight != nullptr) != (grad_pre_weight != nullptr)) return GRPO_ERR_NULL;
    const bool gates = gate && gate_stride != 0;  // one for every row
    if (gate && !gates && !grad_gate) return GRPO_ERR_NULL;
    if (n_tokens > 0) {
        if ((bad = check_rows(residual_out, residual_out_stride, d_model, rt, pre_weight != nullptr)) != GRPO_OK) return bad;
        if ((bad = check_rows(block, block_stride, d_model, dt, block != nullptr)) != GRPO_OK) return bad;
        if ((bad = check_rows(grad_hidden, grad_hidden_stride, d_model, dt, pre_weight != nullptr)) != GRPO_OK) return bad;
        if ((bad = check_rows(grad_residual_out, grad_residual_out_stride, d_model, rt, grad_residual_out || !pre_weight)) != GRPO_OK)
            return bad;
        if ((bad = check_rows(grad_residual, grad_residual_stride, d_model, rt, true)) != GRPO_OK) return bad;
        if ((bad = check_rows(grad_block, grad_block_stride, d_model, dt, block != nullptr)) != GRPO_OK) return bad;
        if (gates || !gate)
            if ((bad = check_rows(grad_gate, grad_gate_stride, d_model, dt, gates)) != GRPO_OK) return bad;
    }
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < grpo_block_norm_workspace_bytes(n_tokens, d_model))
        return GRPO_ERR_WORKSPACE;
    BlockNorm p = block_norm_params(rt, dt, residual_out, residual_out_stride, block, block_stride, post_weight, gate, gate_stride, pre_weight,
                                    n_tokens, d_model, residual_scale, eps);
    const int64_t rb = rt == GRPO_BF16 ? 2 : 4, db = dt == GRPO_BF16 ? 2 : 4;
    p.dh = (const char *)grad_hidden;
    p.dhs = grad_hidden_stride * db;
    p.dxo = (const char *)grad_residual_out;
    p.dxos = grad_residual_out_stride * rb;
    p.dx = (char *)grad_residual;
    p.dxs = grad_residual_stride * rb;
    p.df = (char *)grad_block;
    p.dfs = grad_block_stride * db;
    p.dg = gates ? (char *)grad_gate : nullptr;
    p.dgs = grad_gate_stride * db;
    p.part = (float *)workspace;
    float *gate_row = gate && !gates ? (float *)grad_gate : nullptr;
    hipStream_t st = (hipStream_t)stream;
    if (rt == GRPO_BF16)
        launch_block_norm_bwd<GRPO_BF16, GRPO_BF16>(p, st, grad_post_weight, gate_row, grad_pre_weight, accumulate_grad_weights);
    else if (dt == GRPO_BF16)
        launch_block_norm_bwd<GRPO_F32, GRPO_BF16>(p, st, grad_post_weight, gate_row, grad_pre_weight, accumulate_grad_weights);
    else
        launch_block_norm_bwd<GRPO_F32, GRPO_F32>(p, st, grad_post_weight, gate_row, grad_pre_weight, accumulate_grad_weights);
    return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}

}  // extern "C"
