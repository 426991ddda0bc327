// vie_policy.cu - what a model learns from tokens that were drawn: their
// log-probabilities under full logits, a clipped policy loss with a KL term and
// a loss of preferred over rejected sequences, each with its gradient.
//
// Per row of logits, z the V values, t the row's token, T the temperature:
//   m  = max z,  s = sum_v exp((z_v - m) / T)
//   lp = (z_t - m) / T - log s
//   q  = softmax(z / T),  d lp / d z_v = ([v = t] - q_v) / T
// A row whose token is outside [0, V) has results 0 and its logits are not read.
// All arithmetic is fp32; a bf16 gradient is rounded once.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "vie_api.h"
#include "vie_block.cuh"
#include "vie_device.cuh"
#include "vie_row_softmax.cuh"

namespace vie {

// Terms of the policy loss; `old` NULL: log-probabilities alone.
struct PolicyTerms {
    const float *old_lp, *advantage, *ref_lp;
    float low, high, kl;
};

struct PolicyParams {
    const void *logits;
    const int32_t *tokens;
    const float *lp_in, *stats_in;  // backward alone: log-probability, m and s of each row
    const float *grad;              // backward: weight of each row's loss, or gradient of its log-probability
    float *loss;                    // forward of a policy loss
    float *lp_out;                  // forward
    float *stats_out;               // forward, or NULL
    void *grad_logits;              // backward
    PolicyTerms terms;
    int64_t ld, ld_grad;
    int V;
    float T;
    uint32_t *flag;
};

// What a row's loss is made of besides its logits, read before those.
struct RowTerms {
    float old_lp = 0.0f, advantage = 0.0f, ref_lp = 0.0f, weight = 0.0f;
    template <bool BWD>
    __device__ __forceinline__ void load(const PolicyParams &a, int64_t row) {
        if (a.terms.old_lp != nullptr) {
            old_lp = a.terms.old_lp[row], advantage = a.terms.advantage[row];
            if (a.terms.kl != 0.0f) ref_lp = a.terms.ref_lp[row];
        }
        if (BWD) weight = a.grad[row];
    }
};

// The loss of one token and its derivative by lp:
//   r = exp(lp - old), A the advantage,
//   loss  = -min(r A, clip(r, 1 - low, 1 + high) A) + kl (exp(ref - lp) - (ref - lp) - 1)
//   slope = -A r if r A is the smaller one, else 0, + kl (1 - exp(ref - lp))
// No advantage, no first term, whatever the ratio; the second is +inf where one
// of the two policies alone rules the token out.
__device__ __forceinline__ float2 policy_terms(const PolicyTerms &a, const RowTerms &t, float lp) {
    const float r = expf(lp - t.old_lp), A = t.advantage;
    const float held = r < 1.0f - a.low ? 1.0f - a.low : r > 1.0f + a.high ? 1.0f + a.high : r;  // (NaN stays)
    const float free_ = A == 0.0f ? 0.0f : r * A, bound = A == 0.0f ? 0.0f : held * A;
    float loss = free_ <= bound ? -free_ : -bound, slope = free_ > bound ? 0.0f : -free_;
    if (a.kl != 0.0f) {
        const float x = t.ref_lp - lp, e = expm1f(x);
        loss += a.kl * (e == INFINITY ? INFINITY : e - x);
        slope -= a.kl * e;
    }
    return make_float2(loss, slope);
}

// Log-probabilities and statistics (FWD) or the gradient (BWD) or both, of the
// log-probabilities themselves or of the policy loss.
//
// A row is a cluster's, a slice of it a CTA's; for both, the slice is read again,
// from L2 as long as the slices in progress fit it (vie_row_softmax.cuh).  The
// gradient is the softmax times a number of the row, but for the token's own value,
// which the thread that has written its vector replaces: no barrier in between.
//
// Bound by bytes.  Measured on bf16 logits without empty rows, and as a share of the time
// that a copy of the bytes read and written once would take:
//   log-probabilities  262144 x 2048: 155 us (1.0), 128256 x 2048: 81 (0.96), 20011 x 4096: 34 (0.71)
//   their gradient     151936 x 4096: 372 us (0.98), 128256 x 2048: 156 (1.0), 20011 x 4096: 54 (0.89)
//   both               151936 x 4096: 446 us (0.82), 262144 x 1024: 193 (0.82), 32000 x 4096:
//                      92 (0.84); fp32 151936 x 2048: 426 (0.86); 1000003 x 128: 125 (0.60)
// What is left in the last: each row's exchange, which the CTAs' other rows hide in
// part (64 % of issue slots used, DRAM 59 % busy; DRAM reads 316 MB of 311, the second
// reading comes from L2).  Short rows: a row's chain of token, slice, sum and result,
// of which a CTA has one at a time (CTAs that stay for more rows, with the next token
// read ahead, were slower: 98 us for both at 20011 x 4096, 68 without; prefetching rows
// before their token is known gains 2 %, and loses it where a tenth of them have none).
//
// U vectors in flight per thread, four CTAs per SM: six (loss and gradient of 151936 x
// 4096 bf16, before a row's terms were read ahead: 450 us; eight vectors with three CTAs
// 476, four with five 484, two with eight 561); for log-probabilities alone eight, but
// where a slice leaves much of its last turn empty with them (262144 x 2048 148 us, 152
// with six; 65536 x 4096 75, 78; 20011 x 4096 34, 31; 151936 x 64 in eight slices 6.7, 5.8).

// One CTA's part of a row with a token.
template <typename T, bool FWD, bool BWD, int U>
struct PolicyRow {
    const PolicyParams &a;
    int64_t row;
    int token;
    Slice<T> sl;
    GradSlice<T> out;
    float c;
    RowTerms terms;
    // The thread that the token's vector is: it reads the token's logit before it
    // writes a gradient there (which may be the same place), and afterwards
    // replaces what the loop has written.
    bool here;

    __device__ __forceinline__ PolicyRow(const PolicyParams &a_, int64_t row_, int token_, int log2_slices, int rank)
        : a(a_), row(row_), token(token_), sl(static_cast<const T *>(a.logits) + row * a.ld, a.V, log2_slices, rank),
          out(static_cast<T *>(a.grad_logits) + row * a.ld_grad, sl), c(exponent_factor(a.T)) {
        const int at = token - sl.e0, vec = at >= 0 ? at / Slice<T>::kVec : -1;
        here = vec >= 0 && vec < sl.nv &&
               static_cast<int>(threadIdx.x) ==
                   (vec < sl.lo ? 0 : vec >= sl.hi ? (sl.nv > 1 ? 1 : 0) : (vec - sl.lo) % kRowThreads);
    }
    __device__ __forceinline__ bool live() const { return token >= 0 && token < a.V; }
    __device__ __forceinline__ void write_row(float loss, float lp, float m, float s) const {
        if (a.terms.old_lp != nullptr) a.loss[row] = loss;
        a.lp_out[row] = lp;
        if (a.stats_out != nullptr) {
            a.stats_out[2 * row] = m;
            a.stats_out[2 * row + 1] = s;
        }
    }
    // An empty slot's results.
    __device__ __forceinline__ void write_empty(bool leads) const {
        if (BWD) clear_gradient(sl, out);
        if (leads && token >= a.V) atomicOr(a.flag, kErrTokenIndex);
        if (FWD && leads) write_row(0.0f, 0.0f, 0.0f, 0.0f);
    }
    // This CTA's statistics to sm.part, and the token's logit to *z_token (read while the
    // slice is, and before anything is written).
    __device__ __forceinline__ void measure(RowSmem &sm, float *z_token) {
        T raw;
        if (threadIdx.x == 0) raw = sl.z[token];
        terms.load<BWD>(a, row);
        slice_statistics<T, U, BWD>(sl, c, sm);
        if (threadIdx.x == 0) *z_token = load_value(&raw);
    }
    __device__ __forceinline__ float log_prob(float z_token, float m, float s) const {
        return s == 0.0f ? -INFINITY : (z_token - m) / a.T - logf(s);
    }
    // The gradient, and the row's results if this is the thread that writes them.
    __device__ __forceinline__ void finish(float z_token, float lp, float m, float s, bool leads) const {
        float2 loss = make_float2(0.0f, 1.0f);
        if (a.terms.old_lp != nullptr) loss = policy_terms(a.terms, terms, lp);
        if (BWD) {
            const Exponent e{finite_max(m), c};
            // (a weight of 0 masks a row, whatever its slope)
            const float slope = terms.weight == 0.0f ? 0.0f : terms.weight * loss.y / a.T;
            const float inv = s == 0.0f ? 0.0f : 1.0f / s;
            if (slope == 0.0f) clear_gradient(sl, out);
            else store_softmax<T, U>(sl, out, e, -slope * inv);
            if (here && slope != 0.0f) store_value(out.g + token, slope * (1.0f - e(z_token) * inv));
        }
        if (FWD && leads) write_row(loss.x, lp, m, s);
    }
};

template <typename T, bool FWD, bool BWD, int U>
__global__ void __launch_bounds__(kRowThreads, 4) policy_kernel(const PolicyParams a, int log2_slices) {
    __shared__ RowSmem sm;
    __shared__ float z_shared;
    const int tid = threadIdx.x;
    const int slices = 1 << log2_slices, rank = blockIdx.x & (slices - 1);
    const bool leads = rank == 0 && tid == 0;
    if (FWD && slices > 1) {
        if (tid == 0) sm.init();
        __syncthreads();
        cluster_arrive_relaxed();  // all CTAs of the cluster run and wait, before their memory is written
    }
    griddep_launch_dependents();
    griddep_wait();  // the inputs may come from the kernel before this one

    const int64_t row = blockIdx.x >> log2_slices;
    PolicyRow<T, FWD, BWD, U> r(a, row, a.tokens[row], log2_slices, rank);
    if (FWD && slices > 1) cluster_wait();
    if (!r.live()) {
        r.write_empty(leads);
        return;
    }
    float m, s, z_token = 0.0f, lp = 0.0f;
    if (FWD) {
        r.measure(sm, &z_shared);
        __syncthreads();
        if (slices > 1) {
            if (tid < 32) send_partial(sm, slices, rank, r.c);
            join_partials(a.flag, sm, slices, r.c, &m, &s);
        } else {
            join_warps(sm, r.c, &m, &s);
        }
        z_token = z_shared;
        lp = r.log_prob(z_token, m, s);
    } else {
        m = a.stats_in[2 * row];
        s = a.stats_in[2 * row + 1];
        if (r.here) z_token = load_value(r.sl.z + r.token);
        if (a.terms.old_lp != nullptr) lp = a.lp_in[row];
        r.terms.template load<BWD>(a, row);
    }
    r.finish(z_token, lp, m, s, leads);
}

// CTAs per row of n rows of this many bytes, on so many SMs (four CTAs each).
//
// At most a slice that a CTA can take without losing what it read from L2, or its turn:
// 64 KB of a gradient alone (128256 x 2048 bf16 166 us, in slices of 125 KB 171; 217047 x
// 1500 195, in slices of 106 KB 199), 112 KB of loss and gradient (us with slices of 40 /
// 81 KB, fp32 41353 x 2183: 131 / 123; of 53 / 106, bf16 217047 x 1500: 250 / 233; of 62 /
// 125, 128256 x 1500: 138 / 146).
//
// Among smaller ones, the quickest by what CTAs cost that run in rounds of as many as the
// device has places for, in KB that one of a full round's CTAs reads: a round its slice and
// 24 for the chain of token, slice, sum and result; a last round that is not full by its
// share of the places, but no less than 1 / 1.6 of the slice (what one CTA alone can read);
// an exchange 4.  Clusters of four and more find 24 of 25 places (of 152 SMs: 146 rows in
// four slices already take a second round).  Slices of 12 KB or more, eight for a row
// (sixteen up to kFewRows).
//
// Against the best number of slices, over 800 calls of 1 to 2048 rows of 40 to 1000 KB, rows
// of other calls in between: 1 % slower on average, 17 % at the most (log-probabilities of
// 305 rows of 424 KB: [35.3] us whole, 30.8 in halves, 30.1 in quarters).  (us with 1 / 2 / 4 / 8
// slices, the rule's in brackets: log-probabilities of 620 rows of 217047 bf16 57.0 / [50.9] /
// 52.1 / 59.2, of 300 of 27566 fp32 9.1 / [8.5] / 10.8 / 15.1; loss and gradient of 61 rows of
// 65536 bf16 13.4 / 9.1 / 9.0 / [6.9], of 256 22.3 / [15.7] / 18.2 / 22.4.)
//
// A gradient's rounds wait for nothing: as many slices of 16 KB as an eighth more than one
// round has places for (us with 4 / 8 / 16: 40 rows of 151936 bf16 7.8 / 6.2 / [5.8], 84 of
// 27566 fp32 5.5 / [4.9] / -, 180 of 20011 bf16, which would take 720 CTAs, [4.6] in two, 5.2).
static int slices_of_row(bool fwd, bool bwd, int64_t bytes, int64_t n, int sms) {
    const int64_t places = 4 * static_cast<int64_t>(sms);
    int64_t slices = 1;
    if (!fwd) {
        while (bytes / slices > 64 * 1024 && n * slices < (1 << 30)) slices *= 2;
        while (slices < kMaxSlices && 2 * n * slices <= places + places / 8 && bytes / slices > 16 * 1024) slices *= 2;
        return static_cast<int>(slices);
    }
    if (bwd)
        while (slices < kSlices && bytes / slices > 112 * 1024) slices *= 2;
    int64_t best = slices;
    double least = INFINITY;
    for (; slices <= (n <= kFewRows ? kMaxSlices : kSlices); slices *= 2) {
        if (best != slices && bytes / slices < 12 * 1024) break;
        const int64_t here = slices <= 2 ? places : places * 24 / 25, ctas = n * slices, rest = ctas % here;
        const double kb = static_cast<double>(bytes) / 1024 / slices;
        double cost = static_cast<double>(ctas / here) * (kb + 24) + (slices > 1 ? 4 : 0);
        if (rest > 0) cost += fmax(kb * rest / here, kb / 1.6) + 24;
        if (cost < least) least = cost, best = slices;
    }
    return static_cast<int>(best);
}

template <typename T, bool FWD, bool BWD, int U>
static cudaError_t start_policy(const PolicyParams &p, int64_t n, int slices, cudaStream_t s) {
    auto kernel = policy_kernel<T, FWD, BWD, U>;
    if (FWD && slices > kSlices) {
        static PerDevice prepared;
        const cudaError_t e =
            prepared.once([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1); });
        if (e != cudaSuccess) return e;
    }
    RowLaunch l(n * slices, FWD && slices > 1 ? slices : 0, 0, s);
    return cudaLaunchKernelEx(&l.cfg, kernel, p, log2_of(slices));
}

template <bool FWD, bool BWD>
static vie_status launch_policy(const char *fn, PolicyParams &p, vie_dtype dtype, int64_t n, vie_stream stream) {
    if (n == 0) return VIE_OK;
    cudaError_t e = device_flag_word(&p.flag);
    if (e != cudaSuccess) return fail_cuda(e, fn);
    int sms = 0;
    e = sm_count(&sms);
    if (e != cudaSuccess) return fail_cuda(e, fn);
    const int slices = slices_of_row(FWD, BWD, static_cast<int64_t>(p.V) * dtype_size(dtype), n, sms);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool bf16 = dtype == VIE_DTYPE_BF16;
    if constexpr (FWD && !BWD) {
        // vectors per thread that a slice's turns have room for, with eight in flight and with six
        const int64_t vectors = static_cast<int64_t>(p.V) * dtype_size(dtype) / slices / 16 + 1;
        const int64_t by8 = (vectors + 8 * kRowThreads - 1) / (8 * kRowThreads) * 8;
        const int64_t by6 = (vectors + 6 * kRowThreads - 1) / (6 * kRowThreads) * 6;
        if (10 * by6 > 9 * by8) {
            e = bf16 ? start_policy<__nv_bfloat16, FWD, BWD, 8>(p, n, slices, s)
                     : start_policy<float, FWD, BWD, 8>(p, n, slices, s);
            return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
        }
    }
    e = bf16 ? start_policy<__nv_bfloat16, FWD, BWD, 6>(p, n, slices, s)
             : start_policy<float, FWD, BWD, 6>(p, n, slices, s);
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

static vie_status check_rows(const char *fn, const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                             const int32_t *tokens, float T) {
    if (n < 0 || n > VIE_MANY_MAX)
        return fail(VIE_ERR_INVALID_ARG, "%s: n=%lld outside [0, %d]", fn, static_cast<long long>(n), VIE_MANY_MAX);
    if (V < 1 || V > VIE_DISTILL_V_MAX)
        return fail(VIE_ERR_INVALID_ARG, "%s: V=%lld outside [1, %d]", fn, static_cast<long long>(V), VIE_DISTILL_V_MAX);
    if (!(T > 0.0f) || std::isinf(T))
        return fail(VIE_ERR_INVALID_ARG, "%s: temperature=%g must be positive and finite", fn, static_cast<double>(T));
    if (n > 0 && tokens == nullptr) return fail(VIE_ERR_INVALID_ARG, "%s: NULL buffer", fn);
    if (!aligned_to(tokens, 4)) return fail(VIE_ERR_INVALID_ARG, "%s: buffers must be 4-byte aligned", fn);
    return check_matrix(fn, "logits", logits, dtype, n, V, ld);
}

static vie_status check_floats(const char *fn, int64_t n, const float *p, bool may_be_null = false) {
    if (p == nullptr && n > 0 && !may_be_null) return fail(VIE_ERR_INVALID_ARG, "%s: NULL buffer", fn);
    if (!aligned_to(p, 4)) return fail(VIE_ERR_INVALID_ARG, "%s: buffers must be 4-byte aligned", fn);
    return VIE_OK;
}

// A gradient apart from the logits, or in their place by rows.
static vie_status check_grad(const char *fn, const void *logits, int64_t ld, const void *out_grad, vie_dtype dtype,
                             int64_t n, int64_t V, int64_t ld_grad) {
    if (n > 1 && out_grad == logits && ld_grad != ld)
        return fail(VIE_ERR_INVALID_ARG, "%s: out_grad in place of logits with another row pitch", fn);
    return check_matrix(fn, "out_grad", out_grad, dtype, n, V, ld_grad);
}

static vie_status check_terms(const char *fn, int64_t n, const PolicyTerms &t) {
    vie_status st = check_floats(fn, n, t.old_lp);
    if (st == VIE_OK) st = check_floats(fn, n, t.advantage);
    if (st == VIE_OK) st = check_floats(fn, n, t.ref_lp, true);
    if (st != VIE_OK) return st;
    if (!(t.low >= 0.0f && t.low <= 1.0f) || !(t.high >= 0.0f) || std::isinf(t.high))
        return fail(VIE_ERR_INVALID_ARG, "%s: clip_low=%g outside [0, 1] or clip_high=%g not finite or negative", fn,
                    static_cast<double>(t.low), static_cast<double>(t.high));
    if (!(t.kl >= 0.0f) || std::isinf(t.kl))
        return fail(VIE_ERR_INVALID_ARG, "%s: kl_coef=%g must be finite and not negative", fn, static_cast<double>(t.kl));
    if (t.kl != 0.0f && t.ref_lp == nullptr && n > 0)
        return fail(VIE_ERR_INVALID_ARG, "%s: kl_coef=%g needs ref_logprob", fn, static_cast<double>(t.kl));
    return VIE_OK;
}

// No result where other threads may still read an input.
static vie_status check_apart(const char *fn, std::initializer_list<const float *> results,
                              std::initializer_list<const float *> inputs, const char *what) {
    for (const float *out : results)
        for (const float *in : inputs)
            if (out != nullptr && out == in) return fail(VIE_ERR_INVALID_ARG, "%s: a result in place of %s", fn, what);
    return VIE_OK;
}

// What is written per row while other CTAs may still read the terms of that row.
static vie_status check_results(const char *fn, int64_t n, const PolicyTerms &t, const float *grad_loss,
                                const float *out_loss, const float *out_logprob, const float *out_stats) {
    vie_status st = check_floats(fn, n, out_loss);
    if (st == VIE_OK) st = check_floats(fn, n, out_logprob);
    if (st == VIE_OK) st = check_floats(fn, n, out_stats, true);
    if (st != VIE_OK || n == 0) return st;
    return check_apart(fn, {out_loss, out_logprob, out_stats}, {t.old_lp, t.advantage, t.ref_lp, grad_loss},
                       "old_logprob, advantage, ref_logprob or grad_loss");
}

static PolicyParams rows_of(const void *logits, int64_t V, int64_t ld, const int32_t *tokens, float T) {
    PolicyParams p = {};
    p.logits = logits, p.tokens = tokens, p.ld = ld, p.V = static_cast<int>(V), p.T = T;
    return p;
}

// ---- preference loss ---------------------------------------------------------
//
// Sequence j holds the tokens offsets[j] to offsets[j + 1] - 1; D_j is its sum of
// lp - ref.  Pair p is sequence 2p, the chosen one, and 2p + 1:
//   h    = beta (D_2p - D_2p+1)
//   loss = (1 - e) softplus(-h) + e softplus(h),  e the label smoothing
//   d loss / d lp = beta (e - sigmoid(-h)) for chosen tokens, the negative for
//                   rejected ones, 0 for tokens of no sequence.

struct PreferenceParams {
    const float *lp, *ref;     // forward; ref may be NULL
    const int32_t *offsets;
    const float *margin_in;    // backward alone
    const float *grad_loss;    // backward
    float *loss, *margin_out;  // forward
    float *grad;               // backward
    int64_t n;
    int pairs;
    float beta, smoothing;
    uint32_t *flag;
};

constexpr int kPairCtas = 8;  // of a pair, at most

// The sum of lp - ref over tokens i, i + step, ... below end, as four running sums.
__device__ __forceinline__ float sum_ratios(const PreferenceParams &a, int i, int end, int step) {
    float s[4] = {};
    for (; i + 3 * step < end; i += 4 * step) {
        float v[4], r[4] = {};
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = a.lp[i + u * step];
        if (a.ref != nullptr) {
#pragma unroll
            for (int u = 0; u < 4; ++u) r[u] = a.ref[i + u * step];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] += v[u] - r[u];
    }
    for (; i < end; i += step) s[0] += a.lp[i] - (a.ref != nullptr ? a.ref[i] : 0.0f);
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// A cluster of CTAs of NT threads per pair, whose sums meet in shared memory.  Bound
// by latency: the offsets, the tokens, the exchange, the gradient (loss and gradient of
// 4 pairs of 2 x 300 tokens 2.8 us, of 256 of 2 x 2048 4.5, of one of 2 x 16384 3.9, with
// one CTA 10.9, of one of 2 x 400000 19, with one CTA 215).
template <bool FWD, bool BWD, int NT>
__global__ void __launch_bounds__(NT) preference_kernel(const PreferenceParams a, int ctas) {
    __shared__ float4 sums[NT / 32];
    __shared__ float2 parts[kPairCtas];  // of the pair's CTAs
    const int tid = threadIdx.x, p = blockIdx.x / ctas, rank = blockIdx.x % ctas;
    const int first = rank * NT + tid, step = ctas * NT;  // this thread's place among the pair's
    if (FWD && ctas > 1) cluster_arrive_relaxed();
    griddep_launch_dependents();
    griddep_wait();
    int o[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) o[i] = a.offsets[2 * p + i];
    const int n = static_cast<int>(a.n);
    if (first == 0 && (o[0] < 0 || o[1] < o[0] || o[2] < o[1] || o[2] > n)) atomicOr(a.flag, kErrOffsets);
    o[0] = min(max(o[0], 0), n);
    o[1] = min(max(o[1], o[0]), n);
    o[2] = min(max(o[2], o[1]), n);
    float h;
    if (FWD) {
        float4 d = make_float4(sum_ratios(a, o[0] + first, o[1], step), sum_ratios(a, o[1] + first, o[2], step), 0.0f, 0.0f);
        d = block_sum<NT>(d, sums);
        if (ctas > 1) {
            cluster_wait();  // all CTAs of the pair run, before their memory is written
            if (tid < ctas) *cluster_peer(&parts[rank], tid) = make_float2(d.x, d.y);
            cluster_arrive();
            cluster_wait();
            d.x = d.y = 0.0f;
            for (int i = 0; i < ctas; ++i) d.x += parts[i].x, d.y += parts[i].y;
        }
        h = a.beta * (d.x - d.y);
    } else {
        h = a.margin_in[p];
    }
    if (FWD && first == 0) {
        const float both = log1pf(expf(-fabsf(h)));  // softplus(x) = both + max(x, 0)
        float loss = 0.0f;                           // (h may be infinite: no product of it with 0)
        if (a.smoothing != 1.0f) loss += (1.0f - a.smoothing) * (h < 0.0f ? both - h : both);
        if (a.smoothing != 0.0f) loss += a.smoothing * (h > 0.0f ? both + h : both);
        a.loss[p] = loss;
        a.margin_out[p] = h;
    }
    if (BWD) {
        const float weight = a.grad_loss[p];
        // (a weight of 0 masks a pair, whatever its margin)
        const float slope = weight == 0.0f ? 0.0f : a.beta * weight * (a.smoothing - 1.0f / (1.0f + expf(h)));
        for (int i = o[0] + first; i < o[2]; i += step) a.grad[i] = i < o[1] ? slope : -slope;
        // tokens of no sequence, shared among all pairs
        const int begin = min(max(a.offsets[0], 0), n), end = min(max(a.offsets[2 * a.pairs], 0), n);
        const int64_t all = static_cast<int64_t>(a.pairs) * step;
        const int64_t mine = static_cast<int64_t>(p) * step + first;
        for (int64_t i = mine; i < begin; i += all) a.grad[i] = 0.0f;
        for (int64_t i = end + mine; i < n; i += all) a.grad[i] = 0.0f;
    }
}

template <bool FWD, bool BWD>
static vie_status launch_preference(const char *fn, PreferenceParams &p, vie_stream stream) {
    cudaError_t e = device_flag_word(&p.flag);
    if (e != cudaSuccess) return fail_cuda(e, fn);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (p.pairs == 0) {
        if (BWD && p.n > 0) e = cudaMemsetAsync(p.grad, 0, sizeof(float) * static_cast<size_t>(p.n), s);
        return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
    }
    // Threads for about 8 tokens each where pairs are too few for the chip (256 pairs of
    // 2 x 2048 tokens: 4.5 us with one CTA each, 5.7 with two): up to eight CTAs, of 1024
    // threads where those of 256 would have more than 32 tokens each left.
    const int64_t mean = p.n / p.pairs;
    int ctas = 1;
    while (ctas < kPairCtas && static_cast<int64_t>(p.pairs) * ctas < 256 && mean > ctas * 8 * 256) ctas *= 2;
    const bool wide = p.pairs <= 64 && mean > kPairCtas * 32 * 256;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    cfg.gridDim = dim3(static_cast<unsigned>(p.pairs * ctas));
    cfg.blockDim = dim3(wide ? 1024 : 256);
    cfg.stream = s;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(ctas);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ctas > 1 ? 2 : 1;
    e = wide ? cudaLaunchKernelEx(&cfg, preference_kernel<FWD, BWD, 1024>, p, ctas)
             : cudaLaunchKernelEx(&cfg, preference_kernel<FWD, BWD, 256>, p, ctas);
    return e == cudaSuccess ? VIE_OK : fail_cuda(e, fn);
}

static vie_status check_pairs(const char *fn, int64_t n, const int32_t *offsets, int64_t pairs, float beta,
                              float smoothing) {
    if (n < 0 || n > VIE_PREFERENCE_N_MAX)
        return fail(VIE_ERR_INVALID_ARG, "%s: n=%lld outside [0, %d]", fn, static_cast<long long>(n),
                    VIE_PREFERENCE_N_MAX);
    if (pairs < 0 || pairs > VIE_MANY_MAX)
        return fail(VIE_ERR_INVALID_ARG, "%s: pairs=%lld outside [0, %d]", fn, static_cast<long long>(pairs),
                    VIE_MANY_MAX);
    if (!std::isfinite(beta)) return fail(VIE_ERR_INVALID_ARG, "%s: beta=%g must be finite", fn, static_cast<double>(beta));
    if (!(smoothing >= 0.0f && smoothing <= 1.0f))
        return fail(VIE_ERR_INVALID_ARG, "%s: label_smoothing=%g outside [0, 1]", fn, static_cast<double>(smoothing));
    if (pairs > 0 && offsets == nullptr) return fail(VIE_ERR_INVALID_ARG, "%s: NULL buffer", fn);
    if (!aligned_to(offsets, 4)) return fail(VIE_ERR_INVALID_ARG, "%s: buffers must be 4-byte aligned", fn);
    return VIE_OK;
}

static PreferenceParams pairs_of(int64_t n, const int32_t *offsets, int64_t pairs, float beta, float smoothing) {
    PreferenceParams p = {};
    p.n = n, p.offsets = offsets, p.pairs = static_cast<int>(pairs), p.beta = beta, p.smoothing = smoothing;
    return p;
}

}  // namespace vie

using namespace vie;

extern "C" {

vie_status vie_token_logprobs(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                              const int32_t *tokens, float temperature, float *out_logprob, float *out_stats,
                              vie_stream stream) {
    const char *fn = "vie_token_logprobs";
    vie_status st = check_rows(fn, logits, dtype, n, V, ld, tokens, temperature);
    if (st == VIE_OK) st = check_floats(fn, n, out_logprob);
    if (st == VIE_OK) st = check_floats(fn, n, out_stats, true);
    if (st != VIE_OK) return st;
    PolicyParams p = rows_of(logits, V, ld, tokens, temperature);
    p.lp_out = out_logprob, p.stats_out = out_stats;
    return launch_policy<true, false>(fn, p, dtype, n, stream);
}

vie_status vie_token_logprobs_grad(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                                   const int32_t *tokens, float temperature, const float *stats,
                                   const float *grad_logprob, void *out_grad, int64_t ld_grad, vie_stream stream) {
    const char *fn = "vie_token_logprobs_grad";
    vie_status st = check_rows(fn, logits, dtype, n, V, ld, tokens, temperature);
    if (st == VIE_OK) st = check_floats(fn, n, stats);
    if (st == VIE_OK) st = check_floats(fn, n, grad_logprob);
    if (st == VIE_OK) st = check_grad(fn, logits, ld, out_grad, dtype, n, V, ld_grad);
    if (st != VIE_OK) return st;
    PolicyParams p = rows_of(logits, V, ld, tokens, temperature);
    p.stats_in = stats, p.grad = grad_logprob, p.grad_logits = out_grad, p.ld_grad = ld_grad;
    return launch_policy<false, true>(fn, p, dtype, n, stream);
}

vie_status vie_policy_loss(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                           const int32_t *tokens, float temperature, const float *old_logprob, const float *advantage,
                           const float *ref_logprob, float clip_low, float clip_high, float kl_coef, float *out_loss,
                           float *out_logprob, float *out_stats, vie_stream stream) {
    const char *fn = "vie_policy_loss";
    PolicyParams p = rows_of(logits, V, ld, tokens, temperature);
    p.terms = {old_logprob, advantage, ref_logprob, clip_low, clip_high, kl_coef};
    vie_status st = check_rows(fn, logits, dtype, n, V, ld, tokens, temperature);
    if (st == VIE_OK) st = check_terms(fn, n, p.terms);
    if (st == VIE_OK) st = check_results(fn, n, p.terms, nullptr, out_loss, out_logprob, out_stats);
    if (st != VIE_OK) return st;
    p.loss = out_loss, p.lp_out = out_logprob, p.stats_out = out_stats;
    return launch_policy<true, false>(fn, p, dtype, n, stream);
}

vie_status vie_policy_loss_grad(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                                const int32_t *tokens, float temperature, const float *old_logprob,
                                const float *advantage, const float *ref_logprob, float clip_low, float clip_high,
                                float kl_coef, const float *logprob, const float *stats, const float *grad_loss,
                                void *out_grad, int64_t ld_grad, vie_stream stream) {
    const char *fn = "vie_policy_loss_grad";
    PolicyParams p = rows_of(logits, V, ld, tokens, temperature);
    p.terms = {old_logprob, advantage, ref_logprob, clip_low, clip_high, kl_coef};
    vie_status st = check_rows(fn, logits, dtype, n, V, ld, tokens, temperature);
    if (st == VIE_OK) st = check_terms(fn, n, p.terms);
    if (st == VIE_OK) st = check_floats(fn, n, logprob);
    if (st == VIE_OK) st = check_floats(fn, n, stats);
    if (st == VIE_OK) st = check_floats(fn, n, grad_loss);
    if (st == VIE_OK) st = check_grad(fn, logits, ld, out_grad, dtype, n, V, ld_grad);
    if (st != VIE_OK) return st;
    p.lp_in = logprob, p.stats_in = stats, p.grad = grad_loss, p.grad_logits = out_grad, p.ld_grad = ld_grad;
    return launch_policy<false, true>(fn, p, dtype, n, stream);
}

vie_status vie_policy_loss_step(const void *logits, vie_dtype dtype, int64_t n, int64_t V, int64_t ld,
                                const int32_t *tokens, float temperature, const float *old_logprob,
                                const float *advantage, const float *ref_logprob, float clip_low, float clip_high,
                                float kl_coef, const float *grad_loss, float *out_loss, float *out_logprob,
                                float *out_stats, void *out_grad, int64_t ld_grad, vie_stream stream) {
    const char *fn = "vie_policy_loss_step";
    PolicyParams p = rows_of(logits, V, ld, tokens, temperature);
    p.terms = {old_logprob, advantage, ref_logprob, clip_low, clip_high, kl_coef};
    vie_status st = check_rows(fn, logits, dtype, n, V, ld, tokens, temperature);
    if (st == VIE_OK) st = check_terms(fn, n, p.terms);
    if (st == VIE_OK) st = check_floats(fn, n, grad_loss);
    if (st == VIE_OK) st = check_results(fn, n, p.terms, grad_loss, out_loss, out_logprob, out_stats);
    if (st == VIE_OK) st = check_grad(fn, logits, ld, out_grad, dtype, n, V, ld_grad);
    if (st != VIE_OK) return st;
    p.grad = grad_loss, p.loss = out_loss, p.lp_out = out_logprob, p.stats_out = out_stats;
    p.grad_logits = out_grad, p.ld_grad = ld_grad;
    return launch_policy<true, true>(fn, p, dtype, n, stream);
}

vie_status vie_preference_loss(const float *logprob, const float *ref_logprob, int64_t n, const int32_t *offsets,
                               int64_t pairs, float beta, float label_smoothing, float *out_loss, float *out_margin,
                               vie_stream stream) {
    const char *fn = "vie_preference_loss";
    vie_status st = check_pairs(fn, n, offsets, pairs, beta, label_smoothing);
    if (st == VIE_OK) st = check_floats(fn, n, logprob);
    if (st == VIE_OK) st = check_floats(fn, n, ref_logprob, true);
    if (st == VIE_OK) st = check_floats(fn, pairs, out_loss);
    if (st == VIE_OK) st = check_floats(fn, pairs, out_margin);
    if (st == VIE_OK && pairs > 0) st = check_apart(fn, {out_loss, out_margin}, {logprob, ref_logprob}, "an input");
    if (st != VIE_OK) return st;
    PreferenceParams p = pairs_of(n, offsets, pairs, beta, label_smoothing);
    p.lp = logprob, p.ref = ref_logprob, p.loss = out_loss, p.margin_out = out_margin;
    return launch_preference<true, false>(fn, p, stream);
}

vie_status vie_preference_loss_grad(const float *margin, int64_t n, const int32_t *offsets, int64_t pairs, float beta,
                                    float label_smoothing, const float *grad_loss, float *out_grad,
                                    vie_stream stream) {
    const char *fn = "vie_preference_loss_grad";
    vie_status st = check_pairs(fn, n, offsets, pairs, beta, label_smoothing);
    if (st == VIE_OK) st = check_floats(fn, pairs, margin);
    if (st == VIE_OK) st = check_floats(fn, pairs, grad_loss);
    if (st == VIE_OK) st = check_floats(fn, n, out_grad);
    if (st == VIE_OK && pairs > 0) st = check_apart(fn, {out_grad}, {margin, grad_loss}, "an input");
    if (st != VIE_OK) return st;
    PreferenceParams p = pairs_of(n, offsets, pairs, beta, label_smoothing);
    p.margin_in = margin, p.grad_loss = grad_loss, p.grad = out_grad;
    return launch_preference<false, true>(fn, p, stream);
}

vie_status vie_preference_loss_step(const float *logprob, const float *ref_logprob, int64_t n, const int32_t *offsets,
                                    int64_t pairs, float beta, float label_smoothing, const float *grad_loss,
                                    float *out_loss, float *out_margin, float *out_grad, vie_stream stream) {
    const char *fn = "vie_preference_loss_step";
    vie_status st = check_pairs(fn, n, offsets, pairs, beta, label_smoothing);
    if (st == VIE_OK) st = check_floats(fn, n, logprob);
    if (st == VIE_OK) st = check_floats(fn, n, ref_logprob, true);
    if (st == VIE_OK) st = check_floats(fn, pairs, grad_loss);
    if (st == VIE_OK) st = check_floats(fn, pairs, out_loss);
    if (st == VIE_OK) st = check_floats(fn, pairs, out_margin);
    if (st == VIE_OK) st = check_floats(fn, n, out_grad);
    if (st == VIE_OK && pairs > 0)
        st = check_apart(fn, {out_loss, out_margin, out_grad}, {logprob, ref_logprob, grad_loss}, "an input");
    if (st != VIE_OK) return st;
    PreferenceParams p = pairs_of(n, offsets, pairs, beta, label_smoothing);
    p.lp = logprob, p.ref = ref_logprob, p.grad_loss = grad_loss;
    p.loss = out_loss, p.margin_out = out_margin, p.grad = out_grad;
    return launch_preference<true, true>(fn, p, stream);
}

}  // extern "C"
