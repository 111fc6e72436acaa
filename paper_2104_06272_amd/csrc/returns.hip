// lambda-returns and advantages over sequences of unequal length:
//   G_t = r_t + disc_t ((1 - lambda) V_{t+1} + lambda G_{t+1}),  A_t = G_t - V_t,  which is the recursion
//   A_t = delta_t + disc_t lambda A_{t+1},  delta_t = r_t + disc_t V_{t+1} - V_t,  A = 0 behind the last token.
#include <math.h>
#include "tokens.h"

namespace ank {

struct ReturnsArgs {
    Seqs q;
    const float* reward; const void* value; const uint8_t* done; const float* bootstrap;
    double gamma, lambda;
    float *adv, *ret;
};

__global__ __launch_bounds__(WG) void returns_zero(const int64_t n, float* adv, float* ret)
{
    const int64_t i = (int64_t)blockIdx.x * WG + threadIdx.x;
    if (i < n) { adv[i] = 0.0f; ret[i] = 0.0f; }
}

// a lane per sequence, backwards; sums in 64 bits
template <class E>
__global__ __launch_bounds__(WG) void returns_serial(const ReturnsArgs a)
{
    const int64_t s = (int64_t)blockIdx.x * WG + threadIdx.x;
    if (s >= a.q.count) return;
    const Seq x = sequence(a.q, s);
    const typename E::T* value = static_cast<const typename E::T*>(a.value);
    double vnext = a.bootstrap ? (double)a.bootstrap[s] : 0.0, A = 0.0;
    for (int64_t j = x.n - 1; j >= 0; --j) {
        const int64_t i = x.first + j * x.step;
        const double v = (double)E::get(value + i), disc = a.done && a.done[i] ? 0.0 : a.gamma;
        A = (double)a.reward[i] + disc * vnext - v + disc * a.lambda * A;
        a.adv[i] = (float)A; a.ret[i] = (float)(A + v);
        vnext = v;
    }
}

}  // namespace ank

using namespace ank;

extern "C" size_t anakin_returns_workspace_bytes(int64_t rows, int64_t count)
{
    if (rows < 0 || rows > MAX_ROWS || count < 0 || count > MAX_ROWS) return 0;
    return 256;
}

extern "C" int32_t anakin_lambda_returns(const anakin_sequences* q, const anakin_returns_args* a, void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!a) return fail(ANAKIN_E_INVALID_ARG, "null arguments");
    if (a->rows < 0 || a->rows > MAX_ROWS) return fail(ANAKIN_E_INVALID_ARG, "rows out of range");
    const int32_t rc = check_sequences(q, a->rows);
    if (rc != ANAKIN_OK) return rc;
    if (a->value_type < ANAKIN_TYPE_FP32 || a->value_type > ANAKIN_TYPE_FP16) return fail(ANAKIN_E_INVALID_ARG, "unknown type of the values");
    if (!(a->gamma >= 0.0 && a->gamma <= 1.0) || !(a->lambda_ >= 0.0 && a->lambda_ <= 1.0)) return fail(ANAKIN_E_INVALID_ARG, "gamma and lambda have to lie in [0, 1]");
    if (a->rows > 0 && (!a->d_reward || !a->d_value || !a->d_adv || !a->d_ret)) return fail(ANAKIN_E_INVALID_ARG, "null rewards, values, adv or ret");
    const int32_t rw = check_workspace(d_workspace, workspace_bytes, anakin_returns_workspace_bytes(a->rows, q->count));
    if (rw != ANAKIN_OK) return rw;
    if (a->rows == 0) return ANAKIN_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const ReturnsArgs k{Seqs{q->layout, q->count, q->length, a->rows, q->d_offsets, q->d_lengths}, a->d_reward, a->d_value, a->d_done, a->d_bootstrap,
                        a->gamma, a->lambda_, a->d_adv, a->d_ret};
    hipLaunchKernelGGL(returns_zero, dim3((unsigned)((a->rows + WG - 1) / WG)), dim3(WG), 0, s, a->rows, a->d_adv, a->d_ret);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && q->count > 0) {
        auto f = a->value_type == ANAKIN_TYPE_FP32 ? returns_serial<Fp32> : a->value_type == ANAKIN_TYPE_BF16 ? returns_serial<Bf16> : returns_serial<Fp16>;
        hipLaunchKernelGGL(f, dim3((unsigned)((q->count + WG - 1) / WG)), dim3(WG), 0, s, k);
        e = hipGetLastError();
    }
    return e == hipSuccess ? ANAKIN_OK : fail_hip(e);
}
