// Drafted tokens kept or turned down against the target's probabilities, from given uniforms.
//
//   p, q: softmax of the target's and the draft policy's logits at the trajectory's temperature; x_i the i-th draft
//   x_i stays while u_i q_i(x_i) < p_i(x_i);  at the first that does not, the next token is drawn from max(0, p_i - q_i), and
//   after the last draft from p.  What is kept and drawn is then distributed as the target's own samples are.
//
// All choices go by whole weights w_j = floor(2^31 exp((l_j - max) / T) + 1/2), as action sampling's do: their sums are exact, so that
// neither verdict nor draw depends on how a row is split over threads.  A difference of two distributions is taken in units of
// 2^-40: floor(w_j 2^40 / W) - floor(v_j 2^40 / V).
#include <cmath>
#include <cstdint>

#include "../../include/rlcs.h"
#include "rlcs_device.cuh"
#include "rlcs_weights.cuh"

namespace {

using namespace rlcs_rows;

constexpr double kShareOne = 0x1p40;      // a probability of 1 in a difference

// What is known of a row of logits: maximum and its first place, whole and plain sums of the exponentials, the drafted token's weight.
struct RowStat {
    u64 sum;
    double all;
    float top, drafted;                   // drafted: the token's logit
    uint32_t weight;
    int32_t best;
};

template <typename T> struct VerifyParams {
    const T* logits;
    const T* drafts;
    const int32_t* tokens;
    const int32_t* offsets;
    const float* uniforms;
    const float* draw_uniforms;
    const float* temperature;
    float temperature_all;
    int32_t* out;
    float* log_probs;
    int32_t* accepted;
    RowStat* stats;                       // [2][T]: of the target's rows, of the draft policy's
    int64_t ld, ldd;
    int32_t rows, seqs, A;
};

constexpr int kThreads = 512;

// The trajectory that row t belongs to, -1 where there is none; the rows [begin, end) of it.
template <typename T> __device__ __forceinline__ int seq_of(const VerifyParams<T>& P, int t, int* begin, int* end) {
    int lo = 0, hi = P.seqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (P.offsets[mid] <= t) lo = mid; else hi = mid - 1;
    }
    *begin = max(P.offsets[lo], 0);
    *end = min(P.offsets[lo + 1], P.rows);
    return t >= *begin && t < *end ? lo : -1;
}

template <typename T> __device__ __forceinline__ float temperature_of(const VerifyParams<T>& P, int b) {
    return P.temperature != nullptr ? P.temperature[b] : P.temperature_all;
}

template <typename V> __device__ __forceinline__ V block_total(V v) {
    __shared__ V part[kThreads / 32];
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    V all = 0;
    for (int k = 0; k < kThreads / 32; ++k) all += part[k];
    return all;
}

// One block a row: target rows first, then the draft policy's.
template <typename T>
__global__ void __launch_bounds__(kThreads) verify_rows_kernel(const __grid_constant__ VerifyParams<T> P) {
    const int t = blockIdx.x % P.rows, which = blockIdx.x / P.rows, tid = threadIdx.x;
    int begin, end;
    const int b = seq_of(P, t, &begin, &end);
    if (b < 0 || (which == 1 && t + 1 == end)) return;
    const T* x = which ? P.drafts + t * P.ldd : P.logits + t * P.ld;
    const float inv = inverse_of(temperature_of(P, b));
    __shared__ u64 best;
    if (tid == 0) best = 0;
    float m = -INFINITY;
    int at = P.A;
    for (int j = tid; j < P.A; j += kThreads) {
        const float f = clean(Vec<T>::load(x + j));
        if (f > m) { m = f; at = j; }
    }
    __syncthreads();
    // the largest, and of equals the first: a key that grows with the value and falls with the place
    const uint32_t u = __float_as_uint(m), key = u ^ (((int32_t)u >> 31) | 0x80000000u);
    atomicMax(&best, (u64)key << 32 | (uint32_t)(~at));
    __syncthreads();
    const uint32_t top_key = (uint32_t)(best >> 32), bits = top_key & 0x80000000u ? top_key ^ 0x80000000u : ~top_key;
    const float top = __uint_as_float(bits);
    u64 sum = 0;
    double all = 0.;
    if (top != -INFINITY)
        for (int j = tid; j < P.A; j += kThreads) {
            const float e = expf(scaled(clean(Vec<T>::load(x + j)), top, inv));
            sum += weight_of(e);
            all += (double)e;
        }
    sum = block_total(sum);
    all = block_total(all);
    if (tid != 0) return;
    const int token = t + 1 < end ? P.tokens[t + 1] : -1;
    RowStat s = {sum, all, top, 0.f, 0u, (int32_t)~(uint32_t)best};
    if (token >= 0 && token < P.A && top != -INFINITY) {
        s.drafted = clean(Vec<T>::load(x + token));
        s.weight = weight_of(expf(scaled(s.drafted, top, inv)));
    }
    P.stats[(int64_t)which * P.rows + t] = s;
}

template <typename T> __device__ __forceinline__ bool stays(const VerifyParams<T>& P, int t, bool greedy) {
    const RowStat& p = P.stats[t];
    const int token = P.tokens[t + 1];
    if (token < 0 || token >= P.A || p.sum == 0) return false;
    if (greedy) return token == p.best;
    double v = 1., V = 1.;
    if (P.drafts != nullptr) {
        const RowStat& q = P.stats[P.rows + t];
        v = (double)q.weight;
        V = (double)q.sum;
    }
    return (double)P.uniforms[t] * (v * (double)p.sum) < (double)p.weight * V;
}

// One block a trajectory: its verdict, and the token after the kept ones.
template <typename T>
__global__ void __launch_bounds__(kThreads) verify_draw_kernel(const __grid_constant__ VerifyParams<T> P) {
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int begin = max(P.offsets[b], 0), end = min(P.offsets[b + 1], P.rows);
    if (begin >= end) {
        if (tid == 0) P.accepted[b] = 0;
        return;
    }
    const float temperature = temperature_of(P, b), inv = inverse_of(temperature);
    const bool greedy = !(temperature > 0.f);
    __shared__ int stop;
    if (tid == 0) stop = end - 1;
    __syncthreads();
    for (int t = begin + tid; t < end - 1; t += kThreads)
        if (!stays(P, t, greedy)) atomicMin(&stop, t);
    __syncthreads();
    const int r = stop;
    auto score = [&](int t, float x) {                        // log-probability under the whole softmax
        const RowStat& p = P.stats[t];
        return (float)((double)scaled(x, p.top, inv) - log(p.all));
    };
    for (int t = begin + tid; t < end; t += kThreads) {
        if (t == r) continue;
        P.out[t] = t < r ? P.tokens[t + 1] : -1;
        P.log_probs[t] = t < r ? score(t, P.stats[t].drafted) : -INFINITY;
    }
    const RowStat p = P.stats[r];
    if (tid == 0) P.accepted[b] = r - begin;
    if (p.sum == 0 || greedy) {
        if (tid == 0) {
            P.out[r] = p.sum == 0 ? -1 : p.best;
            P.log_probs[r] = p.sum == 0 ? -INFINITY : score(r, p.top);
        }
        return;
    }
    const T* x = P.logits + r * P.ld;
    const T* y = r + 1 < end && P.drafts != nullptr ? P.drafts + r * P.ldd : nullptr;
    const int turned = r + 1 < end && P.drafts == nullptr ? P.tokens[r + 1] : -1;
    RowStat q = {};
    if (y != nullptr) q = P.stats[P.rows + r];
    const double p_unit = kShareOne / (double)p.sum, q_unit = q.sum > 0 ? kShareOne / (double)q.sum : 0.;
    auto weight = [&](int j, bool plain) -> u64 {
        const uint32_t w = weight_of(expf(scaled(clean(Vec<T>::load(x + j)), p.top, inv)));
        if (plain) return w;
        if (y == nullptr) return j == turned ? 0 : w;
        const u64 share = (u64)((double)w * p_unit);
        const u64 less = q.sum > 0 ? (u64)((double)weight_of(expf(scaled(clean(Vec<T>::load(y + j)), q.top, inv))) * q_unit) : 0;
        return share > less ? share - less : 0;
    };
    // every warp has a share of the row, in order
    const int per = ((P.A + kThreads / 32 - 1) / (kThreads / 32) + 31) / 32 * 32, j0 = min(warp * per, P.A), j1 = min(j0 + per, P.A);
    __shared__ u64 part[kThreads / 32];
    bool plain = y == nullptr && turned < 0;
    u64 total = 0;
    for (int round = 0; round < 2; ++round) {
        u64 mine = 0;
        for (int j = j0 + lane; j < j1; j += 32) mine += weight(j, plain);
        mine = warp_sum(mine);
        __syncthreads();
        if (lane == 0) part[warp] = mine;
        __syncthreads();
        total = 0;
        for (int k = 0; k < kThreads / 32; ++k) total += part[k];
        if (total > 0 || plain) break;
        plain = true;                                         // nothing is left of the difference: the target's own probabilities
    }
    const u64 target = target_of(P.draw_uniforms[b], total);
    u64 before = 0;
    int holder = 0;
    for (; holder < kThreads / 32 - 1 && before + part[holder] <= target; ++holder) before += part[holder];
    if (warp != holder) return;
    for (int base = j0; base < j1; base += 32) {
        const int j = base + lane;
        const u64 w = j < j1 ? weight(j, plain) : 0;
        u64 run = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const u64 up = __shfl_up_sync(~0u, run, o);
            if (lane >= o) run += up;
        }
        const unsigned over = __ballot_sync(~0u, before + run > target);
        if (over) {
            if (lane == __ffs(over) - 1) {
                P.out[r] = j;
                P.log_probs[r] = score(r, clean(Vec<T>::load(x + j)));
            }
            return;
        }
        before += __shfl_sync(~0u, run, 31);
    }
}

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

size_t workspace_of(int64_t rows) { return (size_t)(2 * rows) * sizeof(RowStat) + 16; }

template <typename T>
int verify_run(const T* logits, int64_t ld, const T* drafts, int64_t ldd, const int32_t* tokens, const int32_t* offsets, const float* uniforms,
               const float* draw_uniforms, const float* temperature, float temperature_all, int32_t* out, float* log_probs, int32_t* accepted,
               int64_t rows, int64_t seqs, int64_t A, void* workspace, size_t workspace_bytes, void* stream) {
    if (rows < 0 || seqs < 0 || A < 0 || A > (int64_t(1) << 22) || rows > (int64_t(1) << 24) || seqs > (int64_t(1) << 24)) return RLCS_ERR_SIZE;
    if (seqs == 0) return RLCS_OK;
    if (rows > 0 && (A == 0 || ld < A || (drafts != nullptr && ldd < A))) return RLCS_ERR_SIZE;
    if (rows > 0 && (ld > (int64_t(1) << 40) / rows || ldd > (int64_t(1) << 40) / rows)) return RLCS_ERR_SIZE;
    if (std::isnan(temperature_all)) return RLCS_ERR_ARG;
    if (offsets == nullptr || accepted == nullptr) return RLCS_ERR_NULL;
    if (rows > 0 && (logits == nullptr || tokens == nullptr || uniforms == nullptr || draw_uniforms == nullptr || out == nullptr || log_probs == nullptr))
        return RLCS_ERR_NULL;
    const void* words[] = {tokens, offsets, uniforms, draw_uniforms, temperature, out, log_probs, accepted};
    for (const void* p : words)
        if (!aligned_to(p, 4)) return RLCS_ERR_ALIGN;
    if (!aligned_to(logits, sizeof(T)) || !aligned_to(drafts, sizeof(T))) return RLCS_ERR_ALIGN;
    if (rows > 0 && (workspace == nullptr || workspace_bytes < workspace_of(rows))) return RLCS_ERR_WORKSPACE;
    if (!aligned_to(workspace, 16)) return RLCS_ERR_ALIGN;
    const VerifyParams<T> P = {logits, drafts, tokens, offsets, uniforms, draw_uniforms, temperature, temperature_all, out, log_probs, accepted,
                               static_cast<RowStat*>(workspace), ld, ldd, (int32_t)rows, (int32_t)seqs, (int32_t)A};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (rows > 0) verify_rows_kernel<T><<<(unsigned)(rows * (drafts != nullptr ? 2 : 1)), kThreads, 0, s>>>(P);
    verify_draw_kernel<T><<<(unsigned)seqs, kThreads, 0, s>>>(P);
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

}  // namespace

extern "C" {

size_t rlcs_verify_drafts_workspace_bytes(int64_t T, int64_t B) {
    return T <= 0 || B <= 0 || T > (int64_t(1) << 24) || B > (int64_t(1) << 24) ? 0 : workspace_of(T);
}

int rlcs_verify_drafts(const float* logits, int64_t ld, const float* draft_logits, int64_t ldd, const int32_t* tokens, const int32_t* offsets,
                       const float* uniforms, const float* draw_uniforms, const float* temperature, float temperature_all, int32_t* out_tokens,
                       float* log_probs, int32_t* accepted, int64_t T, int64_t B, int64_t A, void* workspace, size_t workspace_bytes,
                       void* cuda_stream) {
    return verify_run<float>(logits, ld, draft_logits, ldd, tokens, offsets, uniforms, draw_uniforms, temperature, temperature_all, out_tokens,
                             log_probs, accepted, T, B, A, workspace, workspace_bytes, cuda_stream);
}

int rlcs_verify_drafts_bf16(const uint16_t* logits, int64_t ld, const uint16_t* draft_logits, int64_t ldd, const int32_t* tokens,
                            const int32_t* offsets, const float* uniforms, const float* draw_uniforms, const float* temperature,
                            float temperature_all, int32_t* out_tokens, float* log_probs, int32_t* accepted, int64_t T, int64_t B, int64_t A,
                            void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return verify_run<bf16>(reinterpret_cast<const bf16*>(logits), ld, reinterpret_cast<const bf16*>(draft_logits), ldd, tokens, offsets, uniforms,
                            draw_uniforms, temperature, temperature_all, out_tokens, log_probs, accepted, T, B, A, workspace, workspace_bytes,
                            cuda_stream);
}

}  // extern "C"
