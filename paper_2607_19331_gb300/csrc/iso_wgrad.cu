// iso_wgrad.cu -- the weight gradient G = dY^T X_hat from a checkpoint.
#include "iso_train.cuh"

#include <algorithm>

namespace iso {
namespace {

constexpr int WG_T = 64;    // output tile
constexpr int WG_K = 16;    // tokens per step

template <typename T, typename O>
__global__ void __launch_bounds__(256) k_wgrad_simple(const T* dy, long long ldd, const uint8_t* codes,
                                                      long long ldc, const uint8_t* exps, long long lde, O* out,
                                                      long long ldo, int tokens, int M, int N, int accumulate) {
    __shared__ float sa[WG_K][WG_T + 1], sb[WG_K][WG_T + 1];
    const int m0 = blockIdx.y * WG_T, n0 = blockIdx.x * WG_T;
    const int tm = (threadIdx.x >> 4) * 4, tn = (threadIdx.x & 15) * 4;
    float acc[4][4] = {};
    for (int t0 = 0; t0 < tokens; t0 += WG_K) {
        for (int i = threadIdx.x; i < WG_K * WG_T; i += 256) {
            const int k = i / WG_T, j = i % WG_T, t = t0 + k;
            sa[k][j] = t < tokens && m0 + j < M ? to_f32(dy[(long long)t * ldd + m0 + j]) : 0.0f;
            float x = 0.0f;
            if (t < tokens && n0 + j < N)
                x = (float)(int8_t)codes[(long long)t * ldc + n0 + j] *
                    act_scale(exps[(long long)t * lde + (n0 + j) / ISO_ACT_GROUP]);
            sb[k][j] = x;
        }
        __syncthreads();
        for (int k = 0; k < WG_K; ++k)
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 4; ++b) acc[a][b] += sa[k][tm + a] * sb[k][tn + b];
        __syncthreads();
    }
    for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) {
            const int m = m0 + tm + a, n = n0 + tn + b;
            if (m < M && n < N) {
                O* o = out + (long long)m * ldo + n;
                from_f32(accumulate ? to_f32(*o) + acc[a][b] : acc[a][b], *o);
            }
        }
}

int check_wgrad(const iso_mat* dY, const iso_act* pack, const iso_mat* out) {
    ISO_TRY(check_mat(dY));
    ISO_TRY(check_act(pack));
    ISO_TRY(check_mat(out));
    if (dY->rows != pack->rows || out->rows != dY->cols || out->cols != pack->cols) return ISO_ERR_SHAPE;
    return ISO_OK;
}

}  // namespace
}  // namespace iso

using namespace iso;

extern "C" {

int32_t iso_act_wgrad_workspace_size(const iso_mat* dY, const iso_act* pack, const iso_mat* out, size_t* bytes) {
    if (!bytes) return ISO_ERR_ARG;
    ISO_TRY(check_wgrad(dY, pack, out));
    *bytes = 256;
    return ISO_OK;
}

int32_t iso_act_wgrad(const iso_mat* dY, const iso_act* pack, const iso_mat* out, int32_t accumulate,
                      void* workspace, size_t ws_bytes, int32_t* status, void* stream) {
    ISO_TRY(check_wgrad(dY, pack, out));
    if (accumulate != 0 && accumulate != 1) return ISO_ERR_ARG;
    if (share_bytes(bytes_of(out), bytes_of(dY)) || share_bytes(bytes_of(out), codes_of(pack)) ||
        share_bytes(bytes_of(out), exps_of(pack)))
        return ISO_ERR_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (status && cudaMemsetAsync(status, 0, sizeof(int32_t), s) != cudaSuccess) return ISO_ERR_CUDA;
    if (out->rows == 0 || out->cols == 0) return ISO_OK;
    size_t need = 0;
    iso_act_wgrad_workspace_size(dY, pack, out, &need);
    if (!workspace || ws_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return ISO_ERR_WORKSPACE;
    const dim3 grid((unsigned)((out->cols + WG_T - 1) / WG_T), (unsigned)((out->rows + WG_T - 1) / WG_T));
    auto go = [&](auto* tp, auto* op) -> int {
        using T = std::remove_pointer_t<decltype(tp)>;
        using O = std::remove_pointer_t<decltype(op)>;
        TRAIN_LAUNCH((k_wgrad_simple<T, O><<<grid, 256, 0, s>>>(
            static_cast<const T*>(dY->data), dY->ld, static_cast<const uint8_t*>(pack->codes), pack->ld_codes,
            static_cast<const uint8_t*>(pack->exps), pack->ld_exps, static_cast<O*>(out->data), out->ld,
            (int)dY->rows, (int)out->rows, (int)out->cols, accumulate)));
        return ISO_OK;
    };
    using B = __nv_bfloat16;
    if (dY->dtype == ISO_BF16) return out->dtype == ISO_BF16 ? go((B*)nullptr, (B*)nullptr) : go((B*)nullptr, (float*)nullptr);
    return out->dtype == ISO_BF16 ? go((float*)nullptr, (B*)nullptr) : go((float*)nullptr, (float*)nullptr);
}

}  // extern "C"
