// Loss towards the strongest logits of a teacher, and its gradient, from a student's logits [R, A].
//
//   lq = log softmax(l / T) over all A,   p = softmax(teacher / T) over the row's given entries
//   loss = scale * sum_i p_i (log p_i - lq_{id_i}),   d loss / d l_j = scale / T * (exp(lq_j) - sum_{i: id_i = j} p_i)
//
// One read of the logits and one write of the gradient are the floor.
#include <cmath>
#include <cstdint>

#include "../../include/rlcs.h"
#include "rlcs_device.cuh"
#include "rlcs_pair.cuh"
#include "rlcs_rows.cuh"

namespace {

using namespace rlcs_pair;
using namespace rlcs_rows;

template <typename T> struct DistillParams {
    const T* logits;
    const int32_t* ids;
    const float* teacher;
    const uint8_t* mask;
    float* loss;
    T* dlogits;
    int64_t ld, ldd, R;
    int32_t A, K;
    float inv_t, exp2_t, scale;            // 1 / T and log2(e) / T
};

constexpr int kThreads = 512, kMostTop = 1024;

template <typename T>
__global__ void __launch_bounds__(kThreads) distill_block_kernel(const __grid_constant__ DistillParams<T> P) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __shared__ float part[kThreads / 32], weight[kMostTop];
    __shared__ int32_t place[kMostTop];
    auto total = [&](float v) {
        v = warp_sum(v);
        __syncthreads();
        if (lane == 0) part[warp] = v;
        __syncthreads();
        float all = 0.f;
        for (int k = 0; k < kThreads / 32; ++k) all += part[k];
        return all;
    };
    auto most = [&](float v) {             // NaN where there is one
#pragma unroll
        for (int o = 16; o; o >>= 1) v = max_nan(v, __shfl_xor_sync(~0u, v, o));
        __syncthreads();
        if (lane == 0) part[warp] = v;
        __syncthreads();
        float all = -INFINITY;
        for (int k = 0; k < kThreads / 32; ++k) all = max_nan(all, part[k]);
        return all;
    };
    for (int64_t row = blockIdx.x; row < P.R; row += gridDim.x) {
        const T* x = P.logits + row * P.ld;
        T* y = P.dlogits + row * P.ldd;
        float best = -INFINITY;
        for (int i = tid; i < P.K; i += kThreads) {
            const int id = P.ids[row * P.K + i];
            const bool there = id >= 0 && id < P.A;
            place[i] = there ? id : -1;
            weight[i] = there ? P.teacher[row * P.K + i] : -INFINITY;
            best = max_nan(best, weight[i]);
        }
        best = most(best);
        float m = -INFINITY;
        const bool given = best != -INFINITY && (P.mask == nullptr || P.mask[row] != 0);
        if (given)
            for (int j = tid; j < P.A; j += kThreads) m = max_nan(m, Vec<T>::load(x + j));
        m = most(m);
        if (!given || m == -INFINITY) {
            if (tid == 0 && P.loss != nullptr) P.loss[row] = 0.f;
            if (P.dlogits != nullptr)
                for (int j = tid; j < P.A; j += kThreads) Vec<T>::store(y + j, 0.f);
            continue;
        }
        float s = 0.f, z = 0.f;
        for (int j = tid; j < P.A; j += kThreads) s += exp2_of((Vec<T>::load(x + j) - m) * P.exp2_t);
        s = total(s);
        for (int i = tid; i < P.K; i += kThreads)
            if (place[i] >= 0) z += exp2_of((weight[i] - best) * P.exp2_t);
        z = total(z);
        const float log_s = logf(s), log_z = logf(z);
        float loss = 0.f;
        for (int i = tid; i < P.K; i += kThreads) {
            float p = 0.f;
            if (place[i] >= 0) {
                const float t = (weight[i] - best) * P.inv_t - log_z;
                p = expf(t);
                if (p > 0.f || p != p) loss += p * (t - ((Vec<T>::load(x + place[i]) - m) * P.inv_t - log_s));
            }
            weight[i] = p;
        }
        loss = total(loss);
        if (tid == 0 && P.loss != nullptr) P.loss[row] = P.scale * loss;
        if (P.dlogits == nullptr) continue;
        const float unit = P.scale * P.inv_t, inv = z == z ? 1.f / s : z;      // a teacher of NaN: the whole row
        // an entry that several name gets all of their weight
        float mine[kMostTop / kThreads];
        for (int n = 0, i = tid; i < P.K; i += kThreads, ++n) {
            mine[n] = NAN;
            if (place[i] < 0) continue;
            float p = 0.f;
            for (int k = 0; k < P.K; ++k)
                if (place[k] == place[i]) p += weight[k];
            mine[n] = unit * (exp2_of((Vec<T>::load(x + place[i]) - m) * P.exp2_t) * inv - p);
        }
        __syncthreads();
        for (int j = tid; j < P.A; j += kThreads) Vec<T>::store(y + j, unit * inv * exp2_of((Vec<T>::load(x + j) - m) * P.exp2_t));
        __syncthreads();
        for (int n = 0, i = tid; i < P.K; i += kThreads, ++n)
            if (place[i] >= 0) Vec<T>::store(y + place[i], mine[n]);      // all that name an entry have the same value for it
        __syncthreads();
    }
}

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

template <typename T>
int distill_run(const T* logits, int64_t ld, const int32_t* ids, const float* teacher, const uint8_t* mask, float* loss, T* dlogits, int64_t ldd,
                int64_t R, int64_t A, int64_t K, float temperature, float scale, void* stream) {
    if (R < 0 || A < 0 || K < 0 || A > (int64_t(1) << 22) || K > kMostTop || R > (int64_t(1) << 40)) return RLCS_ERR_SIZE;
    if (R == 0) return RLCS_OK;
    if (A == 0 || ld < A || (dlogits != nullptr && ldd < A)) return RLCS_ERR_SIZE;
    if (ld > (int64_t(1) << 40) / R || ldd > (int64_t(1) << 40) / R) return RLCS_ERR_SIZE;
    if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(1.4426950408889634f / temperature) || !std::isfinite(scale)) return RLCS_ERR_ARG;
    if (logits == nullptr || (K > 0 && (ids == nullptr || teacher == nullptr)) || (loss == nullptr && dlogits == nullptr)) return RLCS_ERR_NULL;
    const void* words[] = {ids, teacher, loss};
    for (const void* p : words)
        if (!aligned_to(p, 4)) return RLCS_ERR_ALIGN;
    if (!aligned_to(logits, sizeof(T)) || !aligned_to(dlogits, sizeof(T))) return RLCS_ERR_ALIGN;
    const DistillParams<T> P = {logits, ids, teacher, mask, loss, dlogits, ld, ldd, R, (int32_t)A, (int32_t)K, 1.f / temperature,
                                1.4426950408889634f / temperature, scale};
    const int64_t most = 8 * rlcs_device::limits().sms;
    distill_block_kernel<T><<<(unsigned)(R < most ? R : most), kThreads, 0, static_cast<cudaStream_t>(stream)>>>(P);
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

}  // namespace

extern "C" {

int rlcs_distill_grad(const float* logits, int64_t ld, const int32_t* teacher_ids, const float* teacher_logits, const uint8_t* mask, float* loss,
                      float* dlogits, int64_t ldd, int64_t R, int64_t A, int64_t K, float temperature, float scale, void* cuda_stream) {
    return distill_run<float>(logits, ld, teacher_ids, teacher_logits, mask, loss, dlogits, ldd, R, A, K, temperature, scale, cuda_stream);
}

int rlcs_distill_grad_bf16(const uint16_t* logits, int64_t ld, const int32_t* teacher_ids, const float* teacher_logits, const uint8_t* mask,
                           float* loss, uint16_t* dlogits, int64_t ldd, int64_t R, int64_t A, int64_t K, float temperature, float scale,
                           void* cuda_stream) {
    return distill_run<bf16>(reinterpret_cast<const bf16*>(logits), ld, teacher_ids, teacher_logits, mask, loss, reinterpret_cast<bf16*>(dlogits),
                             ldd, R, A, K, temperature, scale, cuda_stream);
}

}  // extern "C"
