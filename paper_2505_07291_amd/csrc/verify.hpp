// Verification of drafted tokens against the target's probabilities, from given random numbers.  Part of grpo.hip's
// translation unit.
//
//   p_i = softmax(z_i / T) of target row i, q_i the draft's (all on the drafted token where there are no draft logits)
//   draft y_i is accepted iff u_i q_i(y_i) < p_i(y_i), up to the first one, n, that is not
//   then one token: the smallest j with  sum_{l <= j} w_l > v sum_l w_l,  w = max(p_n - q_n, 0), or p_n behind the last draft
//
// verify_rows_k forms, for the drafted positions, maxima and sums of exponentials in fp32 and is bound by reading the logits (96
// responses with 5 drafts of 152064 bf16, 292 MB, of which the caches may hold some: 49 us, 6.0 TB/s).  That is enough for a ratio
// that is not within 2^-15 of its random number (the others are decided in fp64), but not for the token: with sums that are off by
// 1e-7 the border of some of 152064 tokens lies between two orders' results in one row of a hundred.
//
// verify_sums_k forms in fp64 what the token needs, of row n alone: then that is one in 10^8.  It is bound by fp64 arithmetic, 19
// instructions an exponential and nine to what it comes from and is added to, of which the GPU does 1.2e12 a second (29e12 lanes of fma, 33 to
// 35e12 of the others), and by the wait for row n and then for its logits before any can begin: that batch 40 us, of them 24 the former.
// It reads its rows once.  p - q needs the rows' sums S_p and S_q, of which only those in fp32 are known before, rho_0 = S_p / S_q by
// them.  So W = sum of max(e_p - rho_0 e_q, 0) is formed, and B, the sum of e_q where that is positive; with rho, the ratio as it is, W +
// (rho_0 - rho) B is S_p times the sum of max(p - q, 0), but for entries that are on the wrong side by rho_0.  How much those
// can be is summed up too (N), and where it could matter, or little is left of W, the sums are formed again with rho.
//
// verify_pick_k, a workgroup to a response, finds the piece in which the sum crosses, and in it the token (5 to 9 us).  That the rows
// behind a refused draft are read for nothing costs less than to follow it: counted by the workgroups' last one, with what it
// takes to hand sums from one to another inside a launch, that batch took 128 us a call, and takes 92.

namespace __attribute__((visibility("hidden"))) grpo_impl {

constexpr int kVerifyBlock = 256;
constexpr int kMaxDrafts = 64;
constexpr int kMaxChunks = 1024;
constexpr int kVerifySlots = 8;   // vectors of a row that a lane of verify_rows_k holds at a time, where it has as many
constexpr int kSumSlots = 2;      // and one of verify_sums_k
// Workgroups from which on they are given twice the entries each, and again, up to eight times as many.  8 responses with 4 drafts (4800
// workgroups of verify_rows_k at first) take 25.4 us a call, 24.9 from half as many on and 27.7 from twice as many; of verify_sums_k,
// 16 responses with 4 drafts (1200) take 21.9 us, 22.4 from half as many on and 25.4 from twice as many, 32 with 4 40.0, 45.2 and 41.5, and 64
// without drafts, the one that loses, 22.0, 22.4 and 20.4.
constexpr int64_t kRowsEnough = 4096, kSumsEnough = 1024;
// Ratios that fp32 sums do not decide.  A term 2^x of a sum is off by 2^-23 (the instruction) and by the roundings of z - m, of
// 1 / T and of x, 0.7 |x| 2^-24 each, and those below 2^-40 of the largest make up less than 2^-22 of any sum of 2^18 or fewer; three
// roundings in a vector's sum and one of the part's: 94 * 2^-24, under 2^-17, for each of the two rows.
constexpr double kNearRatio = 0x1p-15;
// And entries for which they do not say whether p > q: they are hardly ever off by more.
constexpr double kNearSide = 0x1p-20;
constexpr int kSums = 5;

// Where a response's drafts end: row n, of a draft that is refused or (refused = 0) behind the last; and the rows' maxima.
struct Refusal {
    int n, refused;
    float max_p, max_q;
    double rho;  // rho_0: S_p / S_q by the sums in fp32
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
    int chunks, chunk;              // verify_rows_k: parts of a row, and entries in one (of whole vectors of a whole workgroup)
    int pieces, piece, sum_blocks;  // verify_sums_k: pieces of row n, each a wavefront's, and entries in one; workgroups to a response
    double k, kd;                   // log2(e) / T, of the target and of the draft
    unsigned long long *part;       // [batch][2 drafts][chunks]: target rows, then draft rows; maximum, and sum of exp((z - maximum) / T)
    double *sums;                   // [batch][pieces][kSums]: S_p, S_q, W, B, N of a piece of row n
    float *tops;                    // [batch][pieces]: the maximum that S_p and W are relative to
    Refusal *refusal;               // [batch]
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
    __device__ __forceinline__ unsigned long long *parts(int b, int row) const
    {
        return part + ((long long)b * 2 * drafts + row) * chunks;
    }
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

// The same as they lie in memory.
template <grpo_dtype DT>
__device__ __forceinline__ u32x4 logits_raw(const char *row, long long j, long long to)
{
    constexpr int EPV = Elem<DT>::EPV;
    if (j + EPV <= to) return *(const u32x4 *)(row + j * Elem<DT>::BYTES);
    float z[EPV];
#pragma unroll
    for (int i = 0; i < EPV; ++i) z[i] = j + i < to ? load_elem<DT>(row, j + i) : -INFINITY;
    return pack<DT>(z);
}

// SLOTS vectors of a row for each of `lanes` lanes, neighbours at a time, from entry j0 on.  Where all of them are inside the row the loads
// are under no condition: one that is under one is waited for where it ends, each of the vectors alone.
template <grpo_dtype DT, int SLOTS>
__device__ __forceinline__ void logits_raw(const char *row, long long j0, int lane, int lanes, long long to, u32x4 (&v)[SLOTS])
{
    constexpr int EPV = Elem<DT>::EPV;
    if (j0 + (long long)SLOTS * lanes * EPV <= to) {
        const char *at = row + (j0 + lane * EPV) * Elem<DT>::BYTES;
#pragma unroll
        for (int t = 0; t < SLOTS; ++t) v[t] = *(const u32x4 *)(at + t * lanes * 16);
    } else {
#pragma unroll
        for (int t = 0; t < SLOTS; ++t) v[t] = logits_raw<DT>(row, j0 + (t * lanes + lane) * EPV, to);
    }
}

// 2^x for x <= 0 or little more, to 4e-16 of the value: x = n + f with n whole and |f| <= 1/2, and for 2^f the polynomial of degree
// 10 that agrees with it at the eleven Chebyshev points of [-1/2, 1/2] (one of them 0: 2^0 is 1).  Below 2^-1075 the result is 0,
// for -inf too.  NaN is not carried: a sum's maximum is NaN if one of its terms is (see maximum).  15 fp64 instructions; the
// library function takes some three times as many.
__device__ __forceinline__ double exp2_f64(double x)
{
    constexpr double magic = 0x1.8p52;  // adding it leaves the whole part in the low bits
    x = fmax(x, -1100.0);
    const double r = x + magic;
    const double f = x - (r - magic);
    double q = 0x1.e606343d16a96p-28;
    q = fma(q, f, 0x1.b675bc52c98b0p-24);
    q = fma(q, f, 0x1.62bfd47ecba29p-20);
    q = fma(q, f, 0x1.ffcb540682f51p-17);
    q = fma(q, f, 0x1.430913096c64ap-13);
    q = fma(q, f, 0x1.5d87fe9d7a3b5p-10);
    q = fma(q, f, 0x1.3b2ab6fba1defp-7);
    q = fma(q, f, 0x1.c6b08d703ce4ap-5);
    q = fma(q, f, 0x1.ebfbdff82c598p-3);
    q = fma(q, f, 0x1.62e42fefa3a19p-1);
    q = fma(q, f, 1.0);
    return ldexp(q, (int)(unsigned)__builtin_bit_cast(unsigned long long, r));
}

// The larger one, NaN if either is.
__device__ __forceinline__ float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float wave_maximum(float v)
{
    v = maximum(v, dpp_move<0xB1, 0xf>(v, v));
    v = maximum(v, dpp_move<0x4E, 0xf>(v, v));
    v = maximum(v, dpp_move<0x141, 0xf>(v, v));
    v = maximum(v, dpp_move<0x140, 0xf>(v, v));
    v = maximum(v, dpp_move<0x142, 0xa>(-INFINITY, v));
    v = maximum(v, dpp_move<0x143, 0xc>(-INFINITY, v));
    return as_f32((unsigned)__builtin_amdgcn_readlane((int)as_u32(v), 63));
}

// exp((z - m) / T) with k = log2(e) / T; the difference is exact in fp64, and 1 comes of m itself at any temperature.  A sum is kept
// relative to a maximum m; where nothing has been added yet, or all of it is -inf, the maximum is -inf and 0 stands in for it: every z is -inf
// then and adds 0.
__device__ __forceinline__ double reference(float m) { return m == -INFINITY ? 0.0 : (double)m; }
__device__ __forceinline__ double exp_from(float z, double ref, double k) { return exp2_f64(((double)z - ref) * k); }

// A maximum and a sum relative to it; whatever the sum, NaN if the maximum is +inf or NaN.
struct RowSum {
    float max;
    double sum;
};

// A row's maximum and sum from its parts', by one wavefront.
__device__ __forceinline__ RowSum row_sum(const unsigned long long *part, int chunks, double k)
{
    const int lane = threadIdx.x & 63;
    float m = -INFINITY;
    double s = 0.0;
    for (int c = lane; c < chunks; c += 64) {
        const unsigned long long q = part[c];
        const float part_max = as_f32((unsigned)q), part_sum = as_f32((unsigned)(q >> 32));
        const float top = maximum(m, part_max);
        const double ref = reference(top);
        s = s * exp_from(m, ref, k) + (double)part_sum * exp_from(part_max, ref, k);
        m = top;
    }
    const float top = wave_maximum(m);
    s = wave_sum_dpp(s * exp_from(m, reference(top), k));
    return {top, top < INFINITY ? s : __builtin_nan("")};
}

// What a position's fp32 sums say about its draft, by one wavefront: the rows' sums, p(y) and q(y).
struct Position {
    RowSum p, q;
    double py, qy;
};
template <grpo_dtype DT>
__device__ __forceinline__ Position position(const Verify &p, int b, int i)
{
    Position r;
    const long long y = p.tokens[(long long)b * p.drafts + i];
    const bool in = y >= 0 && y < p.vocab;
    const float zp = in ? load_elem<DT>(p.target_row(b, i), y) : 0.f;
    const float zq = in && p.draft ? load_elem<DT>(p.draft_row(b, i), y) : 0.f;
    r.p = row_sum(p.parts(b, i), p.chunks, p.k);
    r.q = {0.f, 1.0};
    r.py = in ? exp_from(zp, reference(r.p.max), p.k) / r.p.sum : 0.0;
    r.qy = 1.0;
    if (p.draft) {
        r.q = row_sum(p.parts(b, p.drafts + i), p.chunks, p.kd);
        r.qy = in ? exp_from(zq, reference(r.q.max), p.kd) / r.q.sum : 0.0;
    }
    return r;
}
// u q < p, u q >= p, or too near to tell from fp32 sums.  NaN is refused.
enum { kAccepted, kRefused, kNear };
__device__ __forceinline__ int verdict(float u, const Position &r)
{
    const double a = (double)u * r.qy;
    if (a < r.py * (1.0 - kNearRatio)) return kAccepted;
    return a <= r.py * (1.0 + kNearRatio) && r.py > 0.0 ? kNear : kRefused;
}

template <grpo_dtype DT, int SLOTS>
__global__ void __launch_bounds__(kVerifyBlock) verify_rows_k(Verify p)
{
    constexpr int EPV = Elem<DT>::EPV;
    __shared__ float lds_m[kVerifyBlock / 64];
    __shared__ double lds_s[kVerifyBlock / 64];
    const int c = blockIdx.x % p.chunks;
    const int rest = blockIdx.x / p.chunks;
    const int b = rest % p.batch, pos = rest / p.batch;  // positions in order, target and draft rows in turn
    const int i = p.draft ? pos >> 1 : pos;
    const bool of_draft = p.draft && (pos & 1);
    if (i >= p.length(b)) return;
    const char *row = of_draft ? p.draft_row(b, i) : p.target_row(b, i);
    const double k = of_draft ? p.kd : p.k;
    const float kf = (float)k;
    const long long from = (long long)c * p.chunk, to = from + p.chunk < p.vocab ? from + p.chunk : p.vocab;
    float m = -INFINITY;
    double s = 0.0;  // of sums of a vector's terms: long parts lose no more than short ones
    for (long long j0 = from; j0 < to; j0 += kVerifyBlock * EPV * SLOTS) {
        u32x4 v[SLOTS];
        float top = m;
        logits_raw<DT, SLOTS>(row, j0, threadIdx.x, kVerifyBlock, to, v);
#pragma unroll
        for (int t = 0; t < SLOTS; ++t) {
            float z[EPV];
            unpack<DT>(v[t], z);
#pragma unroll
            for (int e = 0; e < EPV; ++e) top = maximum(top, z[e]);
        }
        top = wave_maximum(top);
        const float ref = top == -INFINITY ? 0.f : top;
        s *= exp_from(m, reference(top), k);
#pragma unroll
        for (int t = 0; t < SLOTS; ++t) {
            if (j0 + (long long)t * kVerifyBlock * EPV >= to) break;
            float x[EPV];
            unpack<DT>(v[t], x);
#pragma unroll
            for (int e = 0; e < EPV; ++e) x[e] = __builtin_amdgcn_exp2f((x[e] - ref) * kf);
#pragma unroll
            for (int o = EPV / 2; o > 0; o >>= 1)
#pragma unroll
                for (int e = 0; e < o; ++e) x[e] += x[e + o];
            s += (double)x[0];
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
        for (int w = 1; w < kVerifyBlock / 64; ++w) top = maximum(top, lds_m[w]);
        const double ref = reference(top);
        s = 0.0;
#pragma unroll
        for (int w = 0; w < kVerifyBlock / 64; ++w) s += lds_s[w] * exp_from(lds_m[w], ref, k);
        p.parts(b, of_draft ? p.drafts + i : i)[c] = (unsigned long long)as_u32((float)s) << 32 | as_u32(top);
    }
}

// Sums of the lanes up to and with this one: within rows of 16, then over lane 15 of each row and lane 31.
__device__ __forceinline__ double wave_scan(double v)
{
    v += dpp_move<0x111, 0xf>(v);
    v += dpp_move<0x112, 0xf>(v);
    v += dpp_move<0x114, 0xf>(v);
    v += dpp_move<0x118, 0xf>(v);
    v += dpp_move<0x142, 0xa>(v);
    v += dpp_move<0x143, 0xc>(v);
    return v;
}
// The lane in which scanned sums cross, of those that have any.  The scan adds lanes up in different orders: a sum may cross by a
// rounding in a lane that has nothing, and then it is the last one before it.  Without a crossing, the last that has any.
__device__ __forceinline__ int crossing(unsigned long long cross, unsigned long long any)
{
    const unsigned long long upto = cross ? any & ((cross & -cross) * 2 - 1) : any;
    return 63 - __builtin_clzll(upto ? upto : any);
}
__device__ __forceinline__ double last_lane(double v)
{
    const long long b = __builtin_bit_cast(long long, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)b, 63), hi = (unsigned)__builtin_amdgcn_readlane((int)(b >> 32), 63);
    return __builtin_bit_cast(double, (long long)(((unsigned long long)hi << 32) | lo));
}

// Row n and what is taken off it: e_p = exp((z - max_p) / T) and e_q likewise, w = max(e_p - rho e_q, 0) with rho = S_p / S_q.
struct Weights {
    const char *t, *d;  // d: NULL where there is no draft row
    long long y;        // without a draft row, the token that has all of the draft's mass; -1: none has
    double k, kd, pk, qk, rho;  // pk, qk: the maxima
};

template <grpo_dtype DT>
__device__ __forceinline__ void weights(const Weights &r, long long j, long long to, double (&w)[Elem<DT>::EPV])
{
    constexpr int EPV = Elem<DT>::EPV;
    float z[EPV];
    logits_load<DT>(r.t, j, to, z);
#pragma unroll
    for (int e = 0; e < EPV; ++e) w[e] = j + e == r.y ? 0.0 : exp_from(z[e], r.pk, r.k);
    if (!r.d) return;
    logits_load<DT>(r.d, j, to, z);
#pragma unroll
    for (int e = 0; e < EPV; ++e) w[e] = fmax(fma(-r.rho, exp_from(z[e], r.qk, r.kd), w[e]), 0.0);
}

// S_p, S_q, W, B and N of what a lane has of the entries from .. to; DRAFT: r.d is there.  With max_known S_p and W are relative to r.pk;
// without, to the entries' own maximum m, and there is nothing to take off.  N: an entry is on the wrong side by rho_0 by less than
// |rho / rho_0 - 1| e_p - |w|, for a ratio that is off by no more than kNearSide at most that times max(e_p - |w| / kNearSide, 0).
// Asking for the next entries before these are added up takes 3 us off the batch of 96, one vector at a time where there are two rows
// another 3.
template <grpo_dtype DT, int SLOTS, bool EXACT, bool DRAFT>
__device__ __forceinline__ void lane_sums(const Weights &r, long long from, long long to, bool max_known, float &m, double (&s)[kSums])
{
    constexpr int EPV = Elem<DT>::EPV, GROUP = 64 * EPV * SLOTS;
    const int lane = threadIdx.x & 63;
    double pk = r.pk;
    const auto add = [&](const u32x4 (&zr)[SLOTS], const u32x4 (&dr)[SLOTS], long long j0, bool whole) {
        if (!max_known) {
            float now = m;
#pragma unroll
            for (int t = 0; t < SLOTS; ++t) {
                float z[EPV];
                unpack<DT>(zr[t], z);
#pragma unroll
                for (int e = 0; e < EPV; ++e) now = maximum(now, z[e]);
            }
            now = wave_maximum(now);
            pk = reference(now);
            s[0] *= exp_from(m, pk, r.k);
            m = now;
        }
#pragma unroll
        for (int t = 0; t < SLOTS; ++t) {
            const long long j = j0 + (t * 64 + lane) * EPV;
            if (!whole && j0 + (long long)t * 64 * EPV >= to) break;
            float z[EPV];
            double ep[EPV];
            unpack<DT>(zr[t], z);
#pragma unroll
            for (int e = 0; e < EPV; ++e) {
                ep[e] = exp_from(z[e], pk, r.k);
                s[0] += ep[e];
            }
            if constexpr (DRAFT) {
                unpack<DT>(dr[t], z);
#pragma unroll
                for (int e = 0; e < EPV; ++e) {
                    const double eq = exp_from(z[e], r.qk, r.kd);
                    s[1] += eq;
                    const double w = fma(-r.rho, eq, ep[e]);
                    s[2] += fmax(w, 0.0);
                    if constexpr (!EXACT) {
                        s[3] += w > 0.0 ? eq : 0.0;
                        s[4] += fmax(fma(-1.0 / kNearSide, fabs(w), ep[e]), 0.0);
                    }
                }
            } else if (r.y >= 0) {
#pragma unroll
                for (int e = 0; e < EPV; ++e) s[2] += j + e == r.y ? 0.0 : ep[e];
            }
        }
    };
    u32x4 zr[SLOTS], dr[SLOTS];
    const int groups = (int)((to - from) / GROUP);
    if (groups > 0) {  // the next one is asked for before this one is added up; behind the last, the last again
        const char *zp = r.t + (from + lane * EPV) * Elem<DT>::BYTES, *dp = DRAFT ? r.d + (from + lane * EPV) * Elem<DT>::BYTES : nullptr;
#pragma unroll
        for (int t = 0; t < SLOTS; ++t) {
            zr[t] = *(const u32x4 *)(zp + t * 1024);
            if constexpr (DRAFT) dr[t] = *(const u32x4 *)(dp + t * 1024);
        }
#pragma unroll 1
        for (int g = 0; g < groups; ++g) {
            u32x4 zn[SLOTS], dn[SLOTS];
            const long long next = (long long)(g + 1 < groups ? g + 1 : g) * (GROUP * Elem<DT>::BYTES);
#pragma unroll
            for (int t = 0; t < SLOTS; ++t) {
                zn[t] = *(const u32x4 *)(zp + next + t * 1024);
                if constexpr (DRAFT) dn[t] = *(const u32x4 *)(dp + next + t * 1024);
            }
            add(zr, dr, from + (long long)g * GROUP, true);
#pragma unroll
            for (int t = 0; t < SLOTS; ++t) {
                zr[t] = zn[t];
                if constexpr (DRAFT) dr[t] = dn[t];
            }
        }
    }
    const long long rest = from + (long long)groups * GROUP;
    if (rest < to) {
        logits_raw<DT, SLOTS>(r.t, rest, lane, 64, to, zr);
        if constexpr (DRAFT) logits_raw<DT, SLOTS>(r.d, rest, lane, 64, to, dr);
        add(zr, dr, rest, false);
    }
}

// The same by one wavefront, which all of its lanes get, and top = m.  EXACT: r.rho is S_p / S_q.
template <grpo_dtype DT, int SLOTS, bool EXACT = false>
__device__ __forceinline__ void part_sums(const Weights &r, long long from, long long to, bool max_known, float &top, double (&s)[kSums])
{
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kSums; ++i) s[i] = 0.0;
    if (r.d)
        lane_sums<DT, 1, EXACT, true>(r, from, to, max_known, m, s);
    else
        lane_sums<DT, SLOTS, EXACT, false>(r, from, to, max_known, m, s);
    if (!max_known) top = m;
    s[0] = wave_sum_dpp(s[0]);
    if (!(top < INFINITY)) s[0] = __builtin_nan("");
    if (r.d) {
        s[1] = wave_sum_dpp(s[1]);
        s[3] = wave_sum_dpp(s[3]);
        s[4] = wave_sum_dpp(s[4]);
    }
    if (r.d || r.y >= 0) s[2] = wave_sum_dpp(s[2]);
}

template <grpo_dtype DT, int SLOTS>
__global__ void __launch_bounds__(kVerifyBlock) verify_sums_k(Verify p)
{
    __shared__ Position at[kMaxDrafts];
    __shared__ double whole[kVerifyBlock / 64][2];
    const int b = blockIdx.x / p.sum_blocks, c = blockIdx.x % p.sum_blocks;
    const int tid = threadIdx.x, wave = tid >> 6;
    const int len = p.length(b);
    if (len < 0) return;
    for (int i = wave; i < len; i += kVerifyBlock / 64) {
        const Position r = position<DT>(p, b, i);
        if ((tid & 63) == 0) at[i] = r;
    }
    if (len > 0) __syncthreads();
    Weights r = {};
    r.k = p.k;
    r.kd = p.kd;
    r.y = -1;
    double s[kSums];
    float top = -INFINITY;
    int n = 0;
    for (; n < len; ++n) {
        const float u = p.u[(long long)b * p.drafts + n];
        int said = verdict(u, at[n]);
        if (said == kNear) {  // by the whole rows' sums in fp64, a quarter of them to a wavefront
            const long long y = p.tokens[(long long)b * p.drafts + n], quarter = (p.vocab / 4 + 7) / 8 * 8, from = wave * quarter;
            r.t = p.target_row(b, n);
            r.d = p.draft ? p.draft_row(b, n) : nullptr;
            r.pk = reference(at[n].p.max);
            r.qk = reference(at[n].q.max);
            top = at[n].p.max;
            part_sums<DT, SLOTS>(r, from, wave < 3 && from + quarter < p.vocab ? from + quarter : p.vocab, true, top, s);
            __syncthreads();
            if ((tid & 63) == 0) {
                whole[wave][0] = s[0];
                whole[wave][1] = s[1];
            }
            __syncthreads();
            const double sp = whole[0][0] + whole[1][0] + whole[2][0] + whole[3][0], sq = whole[0][1] + whole[1][1] + whole[2][1] + whole[3][1];
            const double py = exp_from(load_elem<DT>(r.t, y), r.pk, p.k) / sp;
            const double qy = r.d ? exp_from(load_elem<DT>(r.d, y), r.qk, p.kd) / sq : 1.0;
            said = (double)u * qy < py ? kAccepted : kRefused;
        }
        if (said == kRefused) break;
    }
    const bool refused = n < len;
    r.t = p.target_row(b, n);
    r.d = nullptr;
    top = -INFINITY;
    if (refused) {
        top = at[n].p.max;
        r.pk = reference(top);
        if (p.draft) {
            r.d = p.draft_row(b, n);
            r.qk = reference(at[n].q.max);
            r.rho = at[n].p.sum / at[n].q.sum;
        } else {
            r.y = p.tokens[(long long)b * p.drafts + n];
        }
    }
    const int piece = c * (kVerifyBlock / 64) + wave;
    if (piece < p.pieces) {
        const long long from = (long long)piece * p.piece, to = from + p.piece < p.vocab ? from + p.piece : p.vocab;
        part_sums<DT, SLOTS>(r, from, to, refused, top, s);
        if ((tid & 63) == 0) {
            double *sums = p.sums + ((long long)b * p.pieces + piece) * kSums;
#pragma unroll
            for (int i = 0; i < kSums; ++i) sums[i] = s[i];
            p.tops[(long long)b * p.pieces + piece] = top;
        }
    }
    if (c != 0) return;
    if (tid == 0) {
        p.refusal[b] = {n, refused, refused ? at[n].p.max : 0.f, refused ? at[n].q.max : 0.f, r.rho};
        p.accepted_out[b] = n;
    }
    if (tid < n) {
        p.tokens_out[(long long)b * (p.drafts + 1) + tid] = p.tokens[(long long)b * p.drafts + tid];
        p.logprobs_out[(long long)b * (p.drafts + 1) + tid] = (float)log(at[tid].py);
    }
}

// Which piece of row n holds the token, by one wavefront, each lane with its share of the pieces, neighbours.
struct Found {
    int piece;             // -1: there is no token, -2: the sums have to be formed again, with rho as it is here
    double base, target;   // the sum in front of the piece, and the one to cross
    double total;          // S_p
    double pk, rho;
    int whole;             // w is p after all: nothing is left of p - q
};
__device__ __forceinline__ Found find_piece(const Verify &p, int b, const Refusal &at, const Weights &r, bool exact)
{
    const int lane = threadIdx.x & 63;
    const int share = (p.pieces + 63) / 64, first = lane * share, end = first + share < p.pieces ? first + share : p.pieces;
    const double *sums = p.sums + (long long)b * p.pieces * kSums;
    const float *tops = p.tops + (long long)b * p.pieces;
    Found f = {-1, 0.0, 0.0, 0.0, 0.0, 0.0, 0};
    float top = at.max_p;
    if (!at.refused) {  // each piece's sum is relative to its own maximum
        top = -INFINITY;
        for (int i = first; i < end; ++i) top = maximum(top, tops[i]);
        top = wave_maximum(top);
    }
    f.pk = reference(top);
    auto of_p = [&](int i) { return at.refused ? sums[kSums * i] : sums[kSums * i] * exp_from(tops[i], f.pk, p.k); };
    double sp = 0.0, sq = 0.0;
    for (int i = first; i < end; ++i) {
        sp += of_p(i);
        if (r.d) sq += sums[kSums * i + 1];
    }
    const double front = wave_scan(sp);
    f.total = last_lane(front);
    if (r.d) sq = wave_sum_dpp(sq);
    if (!(f.total > 0.0 && top < INFINITY) || (r.d && !(sq > 0.0 && at.max_q < INFINITY))) return f;  // NaN too
    double w = sp, up = front, all = f.total;
    bool whole = !r.d && r.y < 0;
    if (!whole) {
        f.rho = r.d ? f.total / sq : 0.0;
        w = 0.0;
        for (int i = first; i < end; ++i) w += fmax(fma(at.rho - f.rho, sums[kSums * i + 3], sums[kSums * i + 2]), 0.0);
        up = wave_scan(w);
        all = last_lane(up);
        if (r.d && !exact) {
            double near = 0.0;
            for (int i = first; i < end; ++i) near += sums[kSums * i + 4];
            near = wave_sum_dpp(near);
            const double off = fabs(f.rho - at.rho) / f.rho;
            if (!(off <= kNearSide && off * near <= 0x1p-38 * all && all >= 0x1p-10 * f.total)) {
                f.piece = -2;
                return f;
            }
        }
        if (!(all > 0.0)) {
            f.whole = 1;
            whole = true;
            w = sp;
            up = front;
            all = f.total;
        }
    }
    f.target = p.v[b] * all;
    // the first lane whose pieces cross, or, where the number is next to 1 and rounding keeps the sum, the last that has any
    const int owner = crossing(__ballot(up > f.target), __ballot(w > 0.0));
    double run = up - w;
    int piece = -1;
    double base = run;
    if (lane == owner)
        for (int i = first; i < end; ++i) {
            const double x = whole ? of_p(i) : fmax(fma(at.rho - f.rho, sums[kSums * i + 3], sums[kSums * i + 2]), 0.0);
            if (x > 0.0) {
                piece = i;
                base = fmin(run, f.target);  // (up - w of this lane may be above the up of the one before it)
            }
            run += x;
            if (run > f.target) break;
        }
    f.piece = __shfl(piece, owner, 64);
    f.base = __shfl(base, owner, 64);
    return f;
}

template <grpo_dtype DT>
__global__ void __launch_bounds__(kVerifyBlock) verify_pick_k(Verify p)
{
    constexpr int EPV = Elem<DT>::EPV;
    __shared__ Found lds_found;
    __shared__ double lds_wave[2][kVerifyBlock / 64];
    __shared__ int lds_first[2], lds_last;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int K = p.drafts;
    long long *tokens_out = p.tokens_out + (long long)b * (K + 1);
    float *logprobs_out = p.logprobs_out + (long long)b * (K + 1);
    const bool response = p.length(b) >= 0;
    const Refusal at = response ? p.refusal[b] : Refusal{-1, 0, 0.f, 0.f, 0.0};
    if (tid <= K && tid > at.n) {  // (a response that is none has no place n)
        tokens_out[tid] = -1;
        logprobs_out[tid] = 0.f;
    }
    if (!response) {
        if (tid == 0) p.accepted_out[b] = 0;
        return;
    }
    Weights r = {};
    r.k = p.k;
    r.kd = p.kd;
    r.y = -1;
    r.t = p.target_row(b, at.n);
    if (at.refused && p.draft) {
        r.d = p.draft_row(b, at.n);
        r.qk = reference(at.max_q);
    } else if (at.refused) {
        r.y = p.tokens[(long long)b * K + at.n];
    }
    if (wave == 0) {
        const Found f = find_piece(p, b, at, r, false);
        if (lane == 0) {
            lds_found = f;
            lds_first[0] = lds_first[1] = 0x7fffffff;
            lds_last = -1;
        }
    }
    __syncthreads();
    if (lds_found.piece == -2) {
        r.pk = lds_found.pk;
        r.rho = lds_found.rho;
        for (int i = wave; i < p.pieces; i += kVerifyBlock / 64) {
            const long long from = (long long)i * p.piece, to = from + p.piece < p.vocab ? from + p.piece : p.vocab;
            double s[kSums];
            float top = at.max_p;
            part_sums<DT, kSumSlots, true>(r, from, to, true, top, s);
            if (lane == 0) {
                p.sums[((long long)b * p.pieces + i) * kSums + 2] = s[2];
                p.sums[((long long)b * p.pieces + i) * kSums + 3] = 0.0;
            }
        }
        __syncthreads();
        if (wave == 0) {
            const Found f = find_piece(p, b, at, r, true);
            if (lane == 0) lds_found = f;
        }
        __syncthreads();
    }
    const Found f = lds_found;
    if (f.piece < 0) {
        if (tid == 0) {
            tokens_out[at.n] = -1;
            logprobs_out[at.n] = __builtin_nanf("");
        }
        return;
    }
    if (f.whole) {
        r.d = nullptr;
        r.y = -1;
    }
    r.pk = f.pk;
    r.rho = f.rho;
    const long long from = (long long)f.piece * p.piece, to = from + p.piece < p.vocab ? from + p.piece : p.vocab;
    double base = f.base;
    int last = -1, turn = 0;  // this lane's last entry that has a weight
    long long token = -1;
    for (long long j0 = from; j0 < to; j0 += kVerifyBlock * EPV, turn ^= 1) {
        const long long j = j0 + tid * EPV;
        double w[EPV], sum = 0.0;
        weights<DT>(r, j, to, w);
#pragma unroll
        for (int e = 0; e < EPV; ++e) {
            sum += w[e];
            if (w[e] > 0.0) last = (int)(j - from) + e;
        }
        const double up = wave_scan(sum);
        if (lane == 63) lds_wave[turn][wave] = up;
        __syncthreads();
        double before = base;
#pragma unroll
        for (int i = 0; i < kVerifyBlock / 64; ++i) {
            if (i < wave) before += lds_wave[turn][i];
            base += lds_wave[turn][i];
        }
        const unsigned long long cross = __ballot(before + up > f.target), any = __ballot(sum > 0.0);
        // one of the wavefronts crosses, up to rounding
        if (cross && any && before <= f.target && lane == crossing(cross, any)) {
            int first = last;
            double run = fmin(before + (up - sum), f.target);
#pragma unroll
            for (int e = 0; e < EPV; ++e) {
                if (run <= f.target && w[e] > 0.0) first = (int)(j - from) + e;
                run += w[e];
            }
            atomicMin(&lds_first[turn], first);
        }
        __syncthreads();
        if (lds_first[turn] != 0x7fffffff) {
            token = from + lds_first[turn];
            break;
        }
    }
    if (token < 0) {  // the entries, added up in another order, stay below what the piece's sum promised: the last that has any
        atomicMax(&lds_last, last);
        __syncthreads();
        token = from + (lds_last > 0 ? lds_last : 0);
    }
    if (tid == 0) {
        tokens_out[at.n] = token;
        logprobs_out[at.n] = (float)(((double)load_elem<DT>(r.t, token) - f.pk) * p.k * 0.6931471805599453094 - log(f.total));
    }
}

// Entries in a part of a row, and parts: at least `enough` workgroups of kVerifyBlock where the rows are long enough for it, `most` parts
// at most.
static bool verify_cut(int64_t rows, int64_t vocab, int dtype, int64_t enough, int64_t most, int *chunk, int *chunks)
{
    const int64_t unit = kVerifyBlock * (dtype == GRPO_BF16 ? 8 : 4);
    int64_t units = 1;
    while ((vocab + units * unit - 1) / (units * unit) > most) units *= 2;
    while (units < kVerifySlots && rows * ((vocab + unit * units - 1) / (unit * units)) >= enough) units *= 2;
    *chunk = (int)(units * unit);
    *chunks = (int)((vocab + units * unit - 1) / (units * unit));
    return rows * *chunks <= kMaxWorkgroups;
}

// Each kernel with as many vectors to a lane as its parts have: one that looked for more would ask for each under a condition.  8
// responses with 4 drafts take 26 us a call, and 33 with eight vectors to a lane always.
template <grpo_dtype DT>
static void launch_verify(const Verify &p, unsigned row_blocks, unsigned sum_blocks, hipStream_t st)
{
    const dim3 block(kVerifyBlock);
    const int unit = kVerifyBlock * Elem<DT>::EPV;
    if (row_blocks > 0) {
        if (p.chunk == unit)
            hipLaunchKernelGGL((verify_rows_k<DT, 1>), dim3(row_blocks), block, 0, st, p);
        else if (p.chunk == 2 * unit)
            hipLaunchKernelGGL((verify_rows_k<DT, 2>), dim3(row_blocks), block, 0, st, p);
        else if (p.chunk == 4 * unit)
            hipLaunchKernelGGL((verify_rows_k<DT, 4>), dim3(row_blocks), block, 0, st, p);
        else
            hipLaunchKernelGGL((verify_rows_k<DT, kVerifySlots>), dim3(row_blocks), block, 0, st, p);
    }
    if (p.piece * 4 == unit)
        hipLaunchKernelGGL((verify_sums_k<DT, 1>), dim3(sum_blocks), block, 0, st, p);
    else
        hipLaunchKernelGGL((verify_sums_k<DT, kSumSlots>), dim3(sum_blocks), block, 0, st, p);
    hipLaunchKernelGGL((verify_pick_k<DT>), dim3((unsigned)p.batch), block, 0, st, p);
}

// The parts, and where they lie in the workspace; its size, or 0 for sizes that cannot be.
static size_t verify_plan(Verify &p, int64_t batch, int64_t drafts, int64_t vocab, int dtype, uintptr_t ws)
{
    if ((dtype != GRPO_F32 && dtype != GRPO_BF16) || batch < 0 || batch > 0x7fffffffll || drafts < 0 || drafts > kMaxDrafts || vocab <= 0 ||
        vocab > kMaxVocab)
        return 0;
    int sum_chunk;
    if (!verify_cut(batch * 2 * drafts, vocab, dtype, kRowsEnough, kMaxChunks, &p.chunk, &p.chunks) ||
        !verify_cut(batch, vocab, dtype, kSumsEnough, kMaxChunks / 4, &sum_chunk, &p.sum_blocks))
        return 0;
    p.piece = sum_chunk / (kVerifyBlock / 64);
    p.pieces = (int)((vocab + p.piece - 1) / p.piece);
    const uintptr_t begin = ws;
    p.part = (unsigned long long *)ws;
    ws += align_up((size_t)batch * 2 * drafts * p.chunks * 8, 256);
    p.sums = (double *)ws;
    ws += align_up((size_t)batch * p.pieces * kSums * 8, 256);
    p.tops = (float *)ws;
    ws += align_up((size_t)batch * p.pieces * 4, 256);
    p.refusal = (Refusal *)ws;
    ws += align_up((size_t)batch * sizeof(Refusal) + 1, 256);
    return ws - begin;
}

}  // namespace grpo_impl

extern "C" {

size_t grpo_verify_workspace_bytes(int64_t batch, int64_t drafts, int64_t vocab, grpo_dtype dtype_arg)
{
    Verify p;
    return verify_plan(p, batch, drafts, vocab, raw_enum(dtype_arg), 0);
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
    const size_t need = verify_plan(p, batch, drafts, vocab, dtype, (uintptr_t)workspace);
    if (need == 0) return GRPO_ERR_SHAPE;
    // 1 / T has to be a number in fp32 too
    if (!(temperature >= 1e-30 && temperature <= 1e30) || !(draft_temperature >= 1e-30 && draft_temperature <= 1e30)) return GRPO_ERR_PARAM;
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
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need)
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
    p.k = log2e / temperature;
    p.kd = log2e / draft_temperature;
    p.tokens_out = (long long *)tokens_out;
    p.accepted_out = n_accepted_out;
    p.logprobs_out = logprobs_out;
    hipStream_t st = (hipStream_t)stream;
    const unsigned row_blocks = (unsigned)(batch * drafts * (draft_logits ? 2 : 1) * p.chunks), sum_blocks = (unsigned)(batch * p.sum_blocks);
    if (dtype == GRPO_BF16)
        launch_verify<GRPO_BF16>(p, row_blocks, sum_blocks, st);
    else
        launch_verify<GRPO_F32>(p, row_blocks, sum_blocks, st);
    return hipGetLastError() == hipSuccess ? GRPO_OK : GRPO_ERR_HIP;
}

}  // extern "C"
