// Gated delta rule: entry points and argument checks.
#include "cawn_delta.cuh"

namespace cawn {
namespace {

int check(const cawn_delta_params *p)
{
    if (p == nullptr) return CAWN_ERR_NULL_POINTER;
    if (p->struct_size != sizeof(cawn_delta_params)) return CAWN_ERR_INVALID_ARG;
    if (p->B < 1 || p->L < 0 || p->Hk < 1 || p->Hv < 1 || p->Hv % p->Hk != 0 || p->Dk < 1 || p->Dv < 1 || !storage_flags_ok(p->flags))
        return CAWN_ERR_INVALID_ARG;
    if (p->Dk % 8 != 0 || p->Dv % 8 != 0 || p->Dk > 128 || p->Dv > 128) return CAWN_ERR_UNSUPPORTED;
    const int64_t qk = (int64_t)p->Hk * p->Dk, vo = (int64_t)p->Hv * p->Dv;
    const int64_t strides[4] = {p->q_stride, p->k_stride, p->v_stride, p->o_stride};
    for (int i = 0; i < 4; i++)
        if (strides[i] != 0 && (strides[i] < (i < 2 ? qk : vo) || strides[i] % 8 != 0)) return CAWN_ERR_INVALID_ARG;
    if ((int64_t)p->B * p->Hv > 65535ll * 64) return CAWN_ERR_UNSUPPORTED;
    double widest = (double)(qk > vo ? qk : vo);
    for (int i = 0; i < 4; i++)
        if ((double)strides[i] > widest) widest = (double)strides[i];
    // every byte offset must fit 63 bits with room
    if ((double)p->B * (double)p->L * widest > 1.0e17) return CAWN_ERR_UNSUPPORTED;
    return CAWN_OK;
}

DeltaParams fill(const cawn_delta_params *p, const void *q, const void *k, const void *v, const float *g, const float *beta,
                 const float *state_in)
{
    DeltaParams P = {};
    P.q = q; P.k = k; P.v = v; P.g = g; P.beta = beta; P.state_in = state_in;
    P.L = p->L; P.B = p->B; P.Hk = p->Hk; P.Hv = p->Hv; P.Dk = p->Dk; P.Dv = p->Dv; P.scale = p->scale;
    const int64_t qk = (int64_t)p->Hk * p->Dk, vo = (int64_t)p->Hv * p->Dv;
    P.q_stride = p->q_stride != 0 ? p->q_stride : qk;
    P.k_stride = p->k_stride != 0 ? p->k_stride : qk;
    P.v_stride = p->v_stride != 0 ? p->v_stride : vo;
    P.o_stride = p->o_stride != 0 ? p->o_stride : vo;
    return P;
}

// A call without tokens hands the state on.
int pass_state(const cawn_delta_params *p, const float *from, float *to, cudaStream_t st)
{
    if (to == nullptr || to == from) return CAWN_OK;
    const size_t bytes = (size_t)p->B * p->Hv * p->Dv * p->Dk * sizeof(float);
    return status_of(from != nullptr ? cudaMemcpyAsync(to, from, bytes, cudaMemcpyDeviceToDevice, st) : cudaMemsetAsync(to, 0, bytes, st));
}

}  // namespace
}  // namespace cawn

extern "C" int cawn_delta_rule_step(const cawn_delta_params *params, const void *q, const void *k, const void *v, const float *g,
                                    const float *beta, const float *state_in, void *o, float *state_out, void *cuda_stream)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (!all_aligned16(q, k, v, g, beta, state_in, o, state_out)) return CAWN_ERR_MISALIGNED;
    if (params->L == 0) return pass_state(params, state_in, state_out, st);
    if (q == nullptr || k == nullptr || v == nullptr || g == nullptr || beta == nullptr || o == nullptr) return CAWN_ERR_NULL_POINTER;
    DeltaParams P = fill(params, q, k, v, g, beta, state_in);
    P.o = o; P.state_out = state_out;
    return status_of(launch_delta_step(P, params->flags != 0, st));
}

extern "C" int cawn_delta_rule_workspace_bytes(const cawn_delta_params *params, int op, size_t *bytes)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    if (op != CAWN_DELTA_FWD && op != CAWN_DELTA_BWD) return CAWN_ERR_INVALID_ARG;
    if (bytes == nullptr) return CAWN_ERR_NULL_POINTER;
    *bytes = 0;
    return CAWN_OK;
}

extern "C" int cawn_delta_rule_fwd(const cawn_delta_params *params, const void *q, const void *k, const void *v, const float *g,
                                   const float *beta, const float *state_in, void *o, float *state_out, void *workspace,
                                   size_t workspace_bytes, void *cuda_stream)
{
    (void)workspace; (void)workspace_bytes;
    return cawn_delta_rule_step(params, q, k, v, g, beta, state_in, o, state_out, cuda_stream);
}

extern "C" int cawn_delta_rule_bwd(const cawn_delta_params *, const void *, const void *, const void *, const float *, const float *,
                                   const float *, const void *, const float *, void *, void *, void *, float *, float *, float *,
                                   void *, size_t, void *)
{
    return CAWN_ERR_UNSUPPORTED;
}
