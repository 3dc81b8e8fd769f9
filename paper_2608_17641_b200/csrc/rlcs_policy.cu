// Policy loss of given actions from logits [R, A], and its gradient.
//
//   lp = log softmax(l / T),  p_j = exp(lp_j),  H = -sum_j p_j lp_j
//   gain = adv * lp_a,  or  min(rho adv, clip(rho, 1 - eps, 1 + eps) adv)  with rho = exp(lp_a - old)
//   loss = -scale * (gain + c H)
//   d loss / d l_j = scale / T * [ s (p_j - [j = a]) + c p_j (lp_j + H) ],   s = adv, or rho adv where unclipped, or 0
//
// With y_j = l_j - max l, S = sum exp(y_j / T) and U = sum exp(y_j / T) y_j:  lp_j = y_j / T - log S, H = log S - U / (S T),
// and the bracket is p_j (s + c (H - log S) + (c / T) y_j): one multiply-add a logit on top of its exponential.  The maximum is
// taken off before the division, so that a masked logit of the type's lowest value cannot overflow.
#include <cmath>
#include <cstdint>

#include "../../include/rlcs.h"
#include "rlcs_rows.cuh"

namespace {

using namespace rlcs_rows;

template <typename T> struct PolicyParams {
    const T* logits;
    int64_t ld;
    const int32_t* actions;
    const uint8_t* mask;
    const float* advantages;
    const float* old_log_probs;
    float* loss;
    float* log_probs;
    float* entropy;
    T* dlogits;
    int64_t ldd;
    int64_t R;
    int A;
    float inv_t, exp2_t, clip, bonus, scale;       // 1 / T and log2(e) / T
};

constexpr float kLowest = -1.0e30f;      // stands for y = -inf where y multiplies exp(y / T) = 0

__device__ __forceinline__ float exp2_of(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// running maximum with the sums relative to it
struct Stat {
    float m, s, u;
};

// the sums of `a` relative to a maximum m that is not below its own
__device__ __forceinline__ Stat rebase(Stat a, float m, float exp2_t) {
    const float y = fmaxf(a.m - m, kLowest), f = exp2_of(y * exp2_t);
    return Stat{m, a.s * f, f == 0.f ? 0.f : (a.u + a.s * y) * f};            // a NaN stays in s
}

__device__ __forceinline__ Stat join(Stat a, Stat b, float exp2_t) {
    const float m = fmaxf(a.m, b.m);
    if (m == -INFINITY) return Stat{m, a.s + b.s, 0.f};
    const Stat x = rebase(a, m, exp2_t), y = rebase(b, m, exp2_t);
    return Stat{m, x.s + y.s, x.u + y.u};
}

// What the gradient pass needs of a row.
struct RowGrad {
    float c0, c1, inv_s, m, hit;          // dl_j = exp(y / T) * inv_s * (c0 + c1 y), minus `hit` at the action
    bool live;
};

template <typename T>
__device__ __forceinline__ RowGrad finish_row(const PolicyParams<T>& P, int64_t row, Stat st, float xa, bool live, bool write) {
    live = live && st.m != -INFINITY;
    float loss = 0.f, lp = 0.f, h = 0.f, slope = 0.f;
    const float log_s = logf(st.s);
    if (live) {
        lp = (xa - st.m) * P.inv_t - log_s;
        h = log_s - st.u / st.s * P.inv_t;
        if (P.advantages != nullptr) {
            const float adv = P.advantages[row];
            float gain = adv * lp;
            slope = adv;
            if (P.old_log_probs != nullptr) {
                const float ratio = expf(lp - P.old_log_probs[row]);
                const float free_ = ratio * adv, held = fminf(fmaxf(ratio, 1.f - P.clip), 1.f + P.clip) * adv;
                gain = fminf(free_, held);
                slope = free_ <= held ? free_ : 0.f;
            }
            loss = -P.scale * (gain + P.bonus * h);
        }
    }
    if (write) {
        if (P.loss != nullptr) P.loss[row] = loss;
        P.log_probs[row] = lp;
        P.entropy[row] = h;
    }
    RowGrad g;
    g.live = live;
    g.m = st.m;
    g.inv_s = P.inv_t / st.s;
    g.c0 = P.scale * (slope + P.bonus * (h - log_s));
    g.c1 = P.scale * P.bonus * P.inv_t;
    g.hit = P.scale * slope * P.inv_t;
    return g;
}

// One thread group a row: NT threads of a block (a warp, or the whole block).  Two passes over the row, the second
// from L2.
template <typename T, int NT>
__global__ void __launch_bounds__(NT < 256 ? 256 : NT) policy_rows_kernel(const __grid_constant__ PolicyParams<T> P) {
    constexpr int N = Vec<T>::N;
    constexpr int kRows = NT < 256 ? 256 / NT : 1;
    const int tid = threadIdx.x % NT;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / NT; row < P.R; row += (int64_t)gridDim.x * kRows) {
        const T* x = P.logits + row * P.ld;
        const int a = P.actions[row];
        const bool live = (P.mask == nullptr || P.mask[row] != 0) && a >= 0 && a < P.A;
        const Span sp = span_of(x, P.A);
        const int rest = sp.head + sp.vecs * N;
        Stat st = {-INFINITY, 0.f, 0.f};
        float xa = 0.f;
        if (live) {
            xa = Vec<T>::load(x + a);
            for (int i = tid; i < sp.vecs; i += NT) {
                float f[N];
                Vec<T>::unpack(*reinterpret_cast<const uint4*>(x + sp.head + (int64_t)i * N), f);
                float top = -INFINITY;
#pragma unroll
                for (int k = 0; k < N; ++k) top = fmaxf(top, f[k]);
                if (top > st.m) st = rebase(st, top, P.exp2_t);
                if (st.m != -INFINITY) {
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const float y = f[k] - st.m, w = exp2_of(y * P.exp2_t);
                        st.s += w;
                        st.u += w * fmaxf(y, kLowest);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < N; ++k) if (f[k] != f[k]) st.s = f[k];
                }
            }
            for (int i = tid; i < sp.head + P.A - rest; i += NT) {
                const float f = Vec<T>::load(x + (i < sp.head ? i : rest + i - sp.head));
                st = join(st, Stat{f, f == -INFINITY ? 0.f : 1.f, 0.f}, P.exp2_t);
                if (f != f) st.s = f;
            }
        }
#pragma unroll
        for (int o = (NT < 32 ? NT : 32) / 2; o; o >>= 1) {
            const Stat other = {__shfl_xor_sync(~0u, st.m, o), __shfl_xor_sync(~0u, st.s, o), __shfl_xor_sync(~0u, st.u, o)};
            st = join(st, other, P.exp2_t);
        }
        if constexpr (NT > 32) {
            __shared__ Stat part[NT / 32];
            __syncthreads();
            if ((tid & 31) == 0) part[tid >> 5] = st;
            __syncthreads();
            st = part[0];
            for (int k = 1; k < NT / 32; ++k) st = join(st, part[k], P.exp2_t);
        }
        const RowGrad g = finish_row(P, row, st, xa, live, tid == 0);
        if (P.dlogits == nullptr) continue;
        T* y = P.dlogits + row * P.ldd;
        auto grad = [&](float f) {
            const float y = f - g.m, w = exp2_of(y * P.exp2_t);
            return w * g.inv_s * (g.c0 + g.c1 * fmaxf(y, kLowest));
        };
        if (((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(y)) & 15) == 0) {
            for (int i = tid; i < sp.vecs; i += NT) {
                const int at = sp.head + i * N;
                float f[N];
                if (g.live) Vec<T>::unpack(*reinterpret_cast<const uint4*>(x + at), f);
#pragma unroll
                for (int k = 0; k < N; ++k) f[k] = g.live ? grad(f[k]) : 0.f;
                if (g.live && a >= at && a < at + N) {
#pragma unroll
                    for (int k = 0; k < N; ++k) f[k] -= at + k == a ? g.hit : 0.f;
                }
                *reinterpret_cast<uint4*>(y + at) = Vec<T>::pack(f);
            }
            for (int i = tid; i < sp.head + P.A - rest; i += NT) {
                const int j = i < sp.head ? i : rest + i - sp.head;
                Vec<T>::store(y + j, g.live ? grad(Vec<T>::load(x + j)) - (j == a ? g.hit : 0.f) : 0.f);
            }
        } else {
            for (int j = tid; j < P.A; j += NT)
                Vec<T>::store(y + j, g.live ? grad(Vec<T>::load(x + j)) - (j == a ? g.hit : 0.f) : 0.f);
        }
    }
}

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

template <typename T>
int policy_run(const T* logits, int64_t ld, const int32_t* actions, const uint8_t* mask, const float* advantages,
               const float* old_log_probs, float* loss, float* log_probs, float* entropy, T* dlogits, int64_t ldd,
               int64_t R, int64_t A, float temperature, float clip, float entropy_coef, float scale, void* stream) {
    if (R < 0 || A < 0 || A > (int64_t(1) << 22) || R > (int64_t(1) << 40)) return RLCS_ERR_SIZE;
    if (R == 0) return RLCS_OK;
    if (A == 0 || ld < A || (dlogits != nullptr && ldd < A)) return RLCS_ERR_SIZE;
    if (ld > (int64_t(1) << 40) / R || ldd > (int64_t(1) << 40) / R) return RLCS_ERR_SIZE;
    if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(1.4426950408889634f / temperature)) return RLCS_ERR_ARG;
    if (!(clip >= 0.f) || !std::isfinite(entropy_coef) || !std::isfinite(scale)) return RLCS_ERR_ARG;
    if (logits == nullptr || actions == nullptr || log_probs == nullptr || entropy == nullptr) return RLCS_ERR_NULL;
    if ((loss != nullptr || dlogits != nullptr || old_log_probs != nullptr) && advantages == nullptr) return RLCS_ERR_NULL;
    const void* words[] = {actions, advantages, old_log_probs, loss, log_probs, entropy};
    for (const void* p : words)
        if (!aligned_to(p, 4)) return RLCS_ERR_ALIGN;
    if (!aligned_to(logits, sizeof(T)) || !aligned_to(dlogits, sizeof(T))) return RLCS_ERR_ALIGN;
    PolicyParams<T> P = {logits, ld, actions, mask, advantages, old_log_probs, loss, log_probs, entropy, dlogits, ldd, R, (int)A,
                         1.f / temperature, 1.4426950408889634f / temperature, clip, entropy_coef, scale};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (A <= 2048) {
        const int64_t blocks = (R + 7) / 8;
        policy_rows_kernel<T, 32><<<(unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)), 256, 0, s>>>(P);
    } else {
        policy_rows_kernel<T, 512><<<(unsigned)(R < (1 << 20) ? R : (1 << 20)), 512, 0, s>>>(P);
    }
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

}  // namespace

extern "C" {

int rlcs_policy_grad(const float* logits, int64_t ld, const int32_t* actions, const uint8_t* mask, const float* advantages,
                     const float* old_log_probs, float* loss, float* log_probs, float* entropy, float* dlogits, int64_t ldd,
                     int64_t R, int64_t A, float temperature, float clip, float entropy_coef, float scale, void* cuda_stream) {
    return policy_run<float>(logits, ld, actions, mask, advantages, old_log_probs, loss, log_probs, entropy, dlogits, ldd, R, A,
                             temperature, clip, entropy_coef, scale, cuda_stream);
}

int rlcs_policy_grad_bf16(const uint16_t* logits, int64_t ld, const int32_t* actions, const uint8_t* mask, const float* advantages,
                          const float* old_log_probs, float* loss, float* log_probs, float* entropy, uint16_t* dlogits, int64_t ldd,
                          int64_t R, int64_t A, float temperature, float clip, float entropy_coef, float scale, void* cuda_stream) {
    return policy_run<bf16>(reinterpret_cast<const bf16*>(logits), ld, actions, mask, advantages, old_log_probs, loss, log_probs,
                            entropy, reinterpret_cast<bf16*>(dlogits), ldd, R, A, temperature, clip, entropy_coef, scale, cuda_stream);
}

}  // extern "C"
