// Actions drawn from logits [R, A] with temperature, top-k, min-p and top-p, one given uniform a row.
//
// All choices go by whole weights w_j = floor(2^31 exp((l_j - max) / T) + 1/2): their sums are exact in 64-bit integers,
// so the drawn action does not depend on how a row is split over threads, and every comparison of the filters is
// made between the same numbers on every run.
#include <cmath>
#include <cstdint>

#include "../../include/rlcs.h"
#include "rlcs_rows.cuh"

namespace {

using namespace rlcs_rows;
typedef unsigned long long u64;

template <typename T> struct SampleParams {
    const T* logits;
    int64_t ld;
    const float* uniforms;
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    float temperature_all, top_p_all, min_p_all;
    int32_t top_k_all;
    int32_t* actions;
    float* log_probs;
    float* kept_log_probs;
    int64_t R;
    int A;
};

// The logit as compared: NaN counts as -inf (never drawn), -0 as +0.
template <typename T> __device__ __forceinline__ float logit(const T* x, int j) { return fmaxf(Vec<T>::load(x + j), -INFINITY) + 0.f; }

// Unsigned key in the order of the floats.
__device__ __forceinline__ uint32_t key_of(float f) {
    const uint32_t u = __float_as_uint(f);
    return u ^ (((int32_t)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ float exp_rel(float x, float m, float inv_t) { return expf(x == m ? 0.f : (x - m) * inv_t); }

// floor(2^31 e + 1/2) for 0 <= e <= 1: the fraction's 24 bits shifted by the exponent, the last place rounded half up.
__device__ __forceinline__ uint32_t weight_of(float e) {
    const uint32_t u = __float_as_uint(e);
    const int down = 127 - (int)(u >> 23);
    const uint32_t frac = (u << 8) | 0x80000000u;
    return down == 0 ? frac : down > 32 ? 0u : ((frac >> (down - 1)) + 1) >> 1;
}

template <int NT> struct Group {                 // NT threads that share a row: a warp, or a whole block
    int tid;
    u64* scratch;                                // NT / 32 words

    __device__ __forceinline__ u64 sum(u64 v) {
        v = warp_sum(v);
        if constexpr (NT > 32) {
            __syncthreads();
            if ((tid & 31) == 0) scratch[tid >> 5] = v;
            __syncthreads();
            v = 0;
            for (int k = 0; k < NT / 32; ++k) v += scratch[k];
        }
        return v;
    }
    __device__ __forceinline__ uint32_t max(uint32_t v) {
        v = warp_max(v);
        if constexpr (NT > 32) {
            __syncthreads();
            if ((tid & 31) == 0) scratch[tid >> 5] = v;
            __syncthreads();
            v = 0;
            for (int k = 0; k < NT / 32; ++k) v = scratch[k] > v ? (uint32_t)scratch[k] : v;
        }
        return v;
    }
    // this warp's value summed over the warps before it; *all = over all warps
    __device__ __forceinline__ u64 before(u64 v, u64* all) {
        u64 mine = 0, total = v;
        if constexpr (NT > 32) {
            __syncthreads();
            if ((tid & 31) == 0) scratch[tid >> 5] = v;
            __syncthreads();
            total = 0;
            for (int k = 0; k < NT / 32; ++k) {
                if (k == (tid >> 5)) mine = total;
                total += scratch[k];
            }
        }
        *all = total;
        return mine;
    }
};

template <typename T, int NT>
__global__ void __launch_bounds__(NT < 256 ? 256 : NT) sample_rows_kernel(const __grid_constant__ SampleParams<T> P) {
    constexpr int kRows = NT < 256 ? 256 / NT : 1;
    __shared__ u64 scratch[NT / 32];
    Group<NT> group = {(int)threadIdx.x % NT, scratch};
    const int tid = group.tid, lane = tid & 31, A = P.A;
    // a warp's own part of the row, a whole number of 32-element steps
    const int part = ((A + NT - 1) / NT) * 32, lo = (tid >> 5) * part, hi = lo + part < A ? lo + part : A;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / NT; row < P.R; row += (int64_t)gridDim.x * kRows) {
        const T* x = P.logits + row * P.ld;
        const float t = P.temperature != nullptr ? P.temperature[row] : P.temperature_all;
        const int k_asked = P.top_k != nullptr ? P.top_k[row] : P.top_k_all;
        const float p = P.top_p != nullptr ? P.top_p[row] : P.top_p_all;
        float low = P.min_p != nullptr ? P.min_p[row] : P.min_p_all;
        const bool greedy = !(t > 0.f);
        const float inv_t = greedy ? 1.f : 1.f / t;
        int limit = k_asked > 0 && k_asked < A ? k_asked : A;
        if (greedy || p <= 0.f || low > 1.f) limit = 1;
        if (!(low > 0.f) || low > 1.f) low = 0.f;

        uint32_t top_key = 0;
        for (int j = tid; j < A; j += NT) { const uint32_t k = key_of(logit(x, j)); top_key = k > top_key ? k : top_key; }
        top_key = group.max(top_key);
        const float m = __uint_as_float(top_key & 0x80000000u ? top_key ^ 0x80000000u : ~top_key);
        if (m == -INFINITY) {
            if (tid == 0) {
                P.actions[row] = -1;
                P.log_probs[row] = -INFINITY;
                P.kept_log_probs[row] = -INFINITY;
            }
            continue;
        }
        u64 all = 0;
        for (int j = tid; j < A; j += NT) all += weight_of(exp_rel(logit(x, j), m, inv_t));
        all = group.sum(all);

        // kept: every key above `cut`, and the first `ties` of those that equal it (where the weight is not below min-p)
        uint32_t cut = 0;
        int ties = A;
        if (limit < A) {
            cut = limit == 1 ? top_key : 0;
            if (limit > 1)
                for (int b = 31; b >= 0; --b) {
                    const uint32_t next = cut | (1u << b);
                    u64 n = 0;
                    for (int j = tid; j < A; j += NT) n += key_of(logit(x, j)) >= next;
                    if (group.sum(n) >= (u64)limit) cut = next;
                }
            u64 above = 0;
            for (int j = tid; j < A; j += NT) above += key_of(logit(x, j)) > cut;
            ties = limit - (int)group.sum(above);
        }
        auto weight = [&](float f) {
            const float e = exp_rel(f, m, inv_t);
            return e >= low ? weight_of(e) : 0u;
        };
        u64 kept = all;
        if (limit < A || low > 0.f) {
            kept = 0;
            for (int j = tid; j < A; j += NT) { const float f = logit(x, j); kept += key_of(f) > cut ? weight(f) : 0u; }
            kept = group.sum(kept);
            if (limit < A) kept += (u64)ties * weight(__uint_as_float(cut & 0x80000000u ? cut ^ 0x80000000u : ~cut));
        }
        if (p < 1.f && limit > 1) {
            const double enough = (double)p * (double)kept;
            uint32_t c = 0;
            for (int b = 31; b >= 0; --b) {
                const uint32_t next = c | (1u << b);
                u64 n = 0;
                if (next >= cut || limit == A)
                    for (int j = tid; j < A; j += NT) { const float f = logit(x, j); n += key_of(f) >= next ? weight(f) : 0u; }
                else
                    n = ~0ull >> 16;
                n = next >= cut || limit == A ? group.sum(n) : n;
                if ((double)n >= enough) c = next;
            }
            u64 above = 0;
            for (int j = tid; j < A; j += NT) { const float f = logit(x, j); above += key_of(f) > c ? weight(f) : 0u; }
            above = group.sum(above);
            const uint32_t w = weight(__uint_as_float(c & 0x80000000u ? c ^ 0x80000000u : ~c));
            int more = w ? (int)((enough - (double)above) / (double)w) : 0;
            while (more > 0 && (double)(above + (u64)(more - 1) * w) >= enough) --more;
            while (w != 0 && (double)(above + (u64)more * w) < enough) ++more;
            if (c > cut || more < ties || limit == A) ties = more;
            cut = c;
            kept = above + (u64)ties * w;
        }
        const double u = (double)P.uniforms[row];
        u64 target = u > 0. ? (u64)(u * (double)kept) : 0;
        if (target >= kept) target = kept - 1;

        // the action: the first index whose kept weights, summed in index order, pass the target
        u64 ties_all = 0;
        int n = 0;
        for (int j = lo + lane; j < hi; j += 32) n += key_of(logit(x, j)) == cut;
        n = warp_sum(n);
        const int ties_before = (int)group.before((u64)n, &ties_all);
        u64 mine = 0;
        int seen = ties_before;
        for (int base = lo; base < hi; base += 32) {
            const int j = base + lane;
            const float f = j < hi ? logit(x, j) : -INFINITY;
            const uint32_t key = j < hi ? key_of(f) : 0;
            const unsigned tied = __ballot_sync(~0u, j < hi && key == cut);
            const bool in = j < hi && (key > cut || (key == cut && seen + __popc(tied & ((1u << lane) - 1)) < ties));
            mine += in ? weight(f) : 0u;
            seen += __popc(tied);
        }
        mine = warp_sum(mine);
        u64 total = 0;
        u64 sum = group.before(mine, &total);
        if (target >= sum && target < sum + mine) {
            seen = ties_before;
            for (int base = lo; base < hi; base += 32) {
                const int j = base + lane;
                const float f = j < hi ? logit(x, j) : -INFINITY;
                const uint32_t key = j < hi ? key_of(f) : 0;
                const unsigned tied = __ballot_sync(~0u, j < hi && key == cut);
                const bool in = j < hi && (key > cut || (key == cut && seen + __popc(tied & ((1u << lane) - 1)) < ties));
                u64 w = in ? weight(f) : 0u;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const u64 v = __shfl_up_sync(~0u, w, o);
                    w += lane >= o ? v : 0;
                }
                const unsigned past = __ballot_sync(~0u, sum + w > target);
                if (past) {
                    if (lane == __ffs(past) - 1) {
                        const double d = f == m ? 0. : (double)((f - m) * inv_t);
                        P.actions[row] = j;
                        P.log_probs[row] = (float)(d - log((double)all * 0x1p-31));
                        P.kept_log_probs[row] = (float)(d - log((double)kept * 0x1p-31));
                    }
                    break;
                }
                sum += __shfl_sync(~0u, w, 31);
                seen += __popc(tied);
            }
        }
    }
}

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

template <typename T>
int sample_run(const SampleParams<T>& P, int64_t A, void* stream) {
    if (P.R < 0 || A < 0 || A > (int64_t(1) << 22) || P.R > (int64_t(1) << 40)) return RLCS_ERR_SIZE;
    if (P.R == 0) return RLCS_OK;
    if (A == 0 || P.ld < A || P.ld > (int64_t(1) << 40) / P.R) return RLCS_ERR_SIZE;
    if (P.temperature_all != P.temperature_all || P.top_p_all != P.top_p_all || P.min_p_all != P.min_p_all) return RLCS_ERR_ARG;
    if (P.logits == nullptr || P.uniforms == nullptr || P.actions == nullptr || P.log_probs == nullptr || P.kept_log_probs == nullptr)
        return RLCS_ERR_NULL;
    const void* words[] = {P.uniforms, P.temperature, P.top_k, P.top_p, P.min_p, P.actions, P.log_probs, P.kept_log_probs};
    for (const void* p : words)
        if (!aligned_to(p, 4)) return RLCS_ERR_ALIGN;
    if (!aligned_to(P.logits, sizeof(T))) return RLCS_ERR_ALIGN;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (A <= 1024) {
        const int64_t blocks = (P.R + 7) / 8;
        sample_rows_kernel<T, 32><<<(unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)), 256, 0, s>>>(P);
    } else {
        sample_rows_kernel<T, 1024><<<(unsigned)(P.R < (1 << 20) ? P.R : (1 << 20)), 1024, 0, s>>>(P);
    }
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

}  // namespace

extern "C" {

int rlcs_sample_actions(const float* logits, int64_t ld, const float* uniforms, const float* temperature, const int32_t* top_k,
                        const float* top_p, const float* min_p, float temperature_all, int32_t top_k_all, float top_p_all,
                        float min_p_all, int32_t* actions, float* log_probs, float* kept_log_probs, int64_t R, int64_t A,
                        void* cuda_stream) {
    return sample_run<float>({logits, ld, uniforms, temperature, top_k, top_p, min_p, temperature_all, top_p_all, min_p_all, top_k_all,
                              actions, log_probs, kept_log_probs, R, (int)A}, A, cuda_stream);
}

int rlcs_sample_actions_bf16(const uint16_t* logits, int64_t ld, const float* uniforms, const float* temperature,
                             const int32_t* top_k, const float* top_p, const float* min_p, float temperature_all, int32_t top_k_all,
                             float top_p_all, float min_p_all, int32_t* actions, float* log_probs, float* kept_log_probs, int64_t R,
                             int64_t A, void* cuda_stream) {
    return sample_run<bf16>({reinterpret_cast<const bf16*>(logits), ld, uniforms, temperature, top_k, top_p, min_p, temperature_all,
                             top_p_all, min_p_all, top_k_all, actions, log_probs, kept_log_probs, R, (int)A}, A, cuda_stream);
}

}  // extern "C"
