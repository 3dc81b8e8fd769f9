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

__device__ __forceinline__ float grad_of(float x, const RowGrad& g, float exp2_t) {
    const float y = x - g.m;
    return exp2_of(y * exp2_t) * g.inv_s * fmaf(g.c1, fmaxf(y, kLowest), g.c0);
}

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

// One thread group a row: NT threads of a block (a warp, or the whole block).  Two passes over the row, the second from
// L2: a thread takes kAhead vectors at a time, so that enough loads are in flight (one at a time: 57 % of the copy
// bandwidth at 4096 x 131072 bfloat16).
template <typename T, int NT>
__global__ void __launch_bounds__(NT < 256 ? 256 : NT) policy_rows_kernel(const __grid_constant__ PolicyParams<T> P) {
    constexpr int N = Vec<T>::N, kAhead = 4;
    constexpr int kRows = NT < 256 ? 256 / NT : 1;
    const int tid = threadIdx.x % NT;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / NT; row < P.R; row += (int64_t)gridDim.x * kRows) {
        const T* x = P.logits + row * P.ld;
        const int a = P.actions[row];
        const bool live = (P.mask == nullptr || P.mask[row] != 0) && a >= 0 && a < P.A;
        const Span sp = span_of(x, P.A);
        const int rest = sp.head + sp.vecs * N;
        const uint4* body = reinterpret_cast<const uint4*>(x + sp.head);
        Stat st = {-INFINITY, 0.f, 0.f};
        float xa = 0.f;
        if (live) {
            xa = Vec<T>::load(x + a);
            auto take = [&](const float* f, int n) {
                float top = -INFINITY;
#pragma unroll
                for (int k = 0; k < n; ++k) top = fmaxf(top, f[k]);
                if (top > st.m) st = rebase(st, top, P.exp2_t);
                // a group of -inf and NaN ahead of every other logit has no base yet: 0 keeps -inf at weight 0
                const float base = st.m == -INFINITY ? 0.f : st.m;
                float s = 0.f, u = 0.f;
#pragma unroll
                for (int k = 0; k < n; ++k) {
                    const float y = f[k] - base, w = exp2_of(y * P.exp2_t);
                    s += w;
                    u = fmaf(w, fmaxf(y, kLowest), u);
                }
                st.s += s;
                st.u += u;
            };
            int i = tid;
            for (; i + (kAhead - 1) * NT < sp.vecs; i += kAhead * NT) {
                uint4 v[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) v[k] = body[i + k * NT];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    float f[N];
                    Vec<T>::unpack(v[k], f);
                    take(f, N);
                }
            }
            for (; i < sp.vecs; i += NT) {
                float f[N];
                Vec<T>::unpack(body[i], f);
                take(f, N);
            }
            for (int j = tid; j < sp.head + P.A - rest; j += NT) {
                const float f = Vec<T>::load(x + (j < sp.head ? j : rest + j - sp.head));
                take(&f, 1);
            }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
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
        if (((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(y)) & 15) == 0) {
            uint4* out = reinterpret_cast<uint4*>(y + sp.head);
            auto give = [&](int i, const uint4& v) {
                float f[N];
                Vec<T>::unpack(v, f);
#pragma unroll
                for (int k = 0; k < N; ++k) f[k] = grad_of(f[k], g, P.exp2_t);
                const int at = a - sp.head - i * N;
                if (at >= 0 && at < N) {
#pragma unroll
                    for (int k = 0; k < N; ++k) f[k] -= k == at ? g.hit : 0.f;
                }
                out[i] = Vec<T>::pack(f);
            };
            int i = tid;
            if (!g.live) {
                for (; i < sp.vecs; i += NT) out[i] = make_uint4(0, 0, 0, 0);
            } else {
                for (; i + (kAhead - 1) * NT < sp.vecs; i += kAhead * NT) {
                    uint4 v[kAhead];
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) v[k] = body[i + k * NT];
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) give(i + k * NT, v[k]);
                }
                for (; i < sp.vecs; i += NT) give(i, body[i]);
            }
            for (int k = tid; k < sp.head + P.A - rest; k += NT) {
                const int j = k < sp.head ? k : rest + k - sp.head;
                Vec<T>::store(y + j, g.live ? grad_of(Vec<T>::load(x + j), g, P.exp2_t) - (j == a ? g.hit : 0.f) : 0.f);
            }
        } else {
            for (int j = tid; j < P.A; j += NT)
                Vec<T>::store(y + j, g.live ? grad_of(Vec<T>::load(x + j), g, P.exp2_t) - (j == a ? g.hit : 0.f) : 0.f);
        }
    }
}

// Up to 64 actions: one thread a row.  The block brings its rows to shared memory as fp32 (whole 16-byte vectors where rows follow
// one another), a thread walks its own row there, and the gradients leave the same way.  Rows of an even number of actions are
// walked from a place of their own each, so that the threads of a warp meet different banks.
constexpr int kSmallRows = 128, kSmallA = 64;

template <typename T>
__global__ void __launch_bounds__(kSmallRows) policy_small_kernel(const __grid_constant__ PolicyParams<T> P, uint32_t a_mul) {
    constexpr int N = Vec<T>::N;
    extern __shared__ __align__(16) float tile[];
    const int A = P.A, tid = threadIdx.x;
    const int64_t row0 = (int64_t)blockIdx.x * kSmallRows, row = row0 + tid;
    const int rows = P.R - row0 < kSmallRows ? (int)(P.R - row0) : kSmallRows, n = rows * A;
    const T* from = P.logits + row0 * P.ld;
    T* to = P.dlogits != nullptr ? P.dlogits + row0 * P.ldd : nullptr;
    auto of = [&](int i) { return a_mul != 0 ? (int)__umulhi((uint32_t)i, a_mul) : i; };      // the row of flat element i
    if (P.ld == A && (reinterpret_cast<uintptr_t>(from) & 15) == 0) {
#pragma unroll 4
        for (int i = tid * N; i < n - N + 1; i += kSmallRows * N) {
            float f[N];
            Vec<T>::unpack(*reinterpret_cast<const uint4*>(from + i), f);
#pragma unroll
            for (int k = 0; k < N; k += 4) *reinterpret_cast<float4*>(tile + i + k) = make_float4(f[k], f[k + 1], f[k + 2], f[k + 3]);
        }
        for (int i = n / N * N + tid; i < n; i += kSmallRows) tile[i] = Vec<T>::load(from + i);
    } else {
#pragma unroll 4
        for (int i = tid; i < n; i += kSmallRows) {
            const int r = of(i);
            tile[i] = Vec<T>::load(from + r * P.ld + (i - r * A));
        }
    }
    __syncthreads();
    if (tid < rows) {
        float* x = tile + tid * A;
        const int a = P.actions[row];
        const bool live = (P.mask == nullptr || P.mask[row] != 0) && a >= 0 && a < A;
        const int first = A & 1 ? 0 : tid % A;
        // every element once, from the thread's own place on
        auto each = [&](auto f) {
#pragma unroll 4
            for (int j = first; j < A; ++j) f(j);
#pragma unroll 4
            for (int j = 0; j < first; ++j) f(j);
        };
        Stat st = {-INFINITY, 0.f, 0.f};
        float xa = 0.f;
        if (live) {
            xa = x[a];
            each([&](int j) { st.m = fmaxf(st.m, x[j]); });
            const float base = st.m == -INFINITY ? 0.f : st.m;
            each([&](int j) {
                const float y = x[j] - base, w = exp2_of(y * P.exp2_t);
                st.s += w;
                st.u = fmaf(w, fmaxf(y, kLowest), st.u);
            });
        }
        const RowGrad g = finish_row(P, row, st, xa, live, true);
        if (to != nullptr) {
            each([&](int j) { x[j] = g.live ? grad_of(x[j], g, P.exp2_t) : 0.f; });
            if (g.live) x[a] -= g.hit;
        }
    }
    if (to == nullptr) return;
    __syncthreads();
    if (P.ldd == A && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
#pragma unroll 4
        for (int i = tid * N; i < n - N + 1; i += kSmallRows * N) {
            float f[N];
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                const float4 v = *reinterpret_cast<const float4*>(tile + i + k);
                f[k] = v.x; f[k + 1] = v.y; f[k + 2] = v.z; f[k + 3] = v.w;
            }
            *reinterpret_cast<uint4*>(to + i) = Vec<T>::pack(f);
        }
        for (int i = n / N * N + tid; i < n; i += kSmallRows) Vec<T>::store(to + i, tile[i]);
    } else {
#pragma unroll 4
        for (int i = tid; i < n; i += kSmallRows) {
            const int r = of(i);
            Vec<T>::store(to + r * P.ldd + (i - r * A), tile[i]);
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
    if (A <= kSmallA) {
        const int64_t blocks = (R + kSmallRows - 1) / kSmallRows;
        if (blocks > (int64_t(1) << 31) - 1) return RLCS_ERR_SIZE;
        const uint32_t mul = A > 1 ? (uint32_t)(((uint64_t(1) << 32) + A - 1) / A) : 0;
        policy_small_kernel<T><<<(unsigned)blocks, kSmallRows, kSmallRows * A * sizeof(float), s>>>(P, mul);
    } else if (A <= 2048) {
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
