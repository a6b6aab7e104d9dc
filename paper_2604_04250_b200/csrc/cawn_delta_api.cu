// Gated delta rule: entry points and argument checks.
#include "cawn_delta_chunk.cuh"

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

// Calls of up to this many tokens run token by token.  Step / chunk, us: bfloat16, 12 heads of 64 x 64, 12 tokens
// 14 / 13, 17 tokens 16 / 13, 24 tokens 21 / 13; 1024 heads of 128 x 128, 17 tokens 107 / 110, 24 tokens 143 / 112.  Float
// storage, whose chunks multiply three terms: 12 heads, 33 tokens 25 / 22, 64 tokens 43 / 22; 1024 heads, 33 tokens 199 / 347,
// 64 tokens 369 / 378.
inline int step_tokens(const cawn_delta_params *p) { return p->flags != 0 ? 16 : 32; }

// The workspace, front to back; sizes in bytes, every part a multiple of 256.
struct Plan {
    int dk, terms, chunks, vblocks, segs, seg_chunks;    // terms: of an input
    size_t q, k, v, go;                  // three bfloat16 terms each, float storage only
    size_t coef, tri, p;
    size_t r, s0, rbt;                  // backward: r also for D K^T, s0 for the adjoints
    size_t seg_state, seg_map;
    size_t total;
};

inline size_t part(double bytes) { return ((size_t)bytes + 255) / 256 * 256; }

Plan plan_of(const cawn_delta_params *p, bool backward)
{
    Plan w = {};
    w.dk = p->Dk <= 64 ? 64 : 128;
    w.terms = p->flags != 0 ? 1 : 3;
    const double nt = w.terms == 1 ? 2 : 3;      // terms of what is computed
    w.chunks = (int)((p->L + kC - 1) / kC);
    w.vblocks = (p->Dv + kC - 1) / kC;
    // Time segments where the heads alone leave SMs without a block.  They cost a second walk over values and keys and
    // the join, so three pay in a forward for long sequences alone.  Three / one, us: forward, 49 heads of 64 in bfloat16 x
    // 1024 tokens 65 / 60, x 2048 99 / 108, x 4096 175 / 200; 24 of 128 97 / 75, 146 / 138, 247 / 263; 24 of 64 in
    // float 103 / 95, 175 / 179, 323 / 349.  Backward, 24 of 64 in bfloat16 x 1024 116 / 114, x 2048 183 / 196; 12 of 128
    // 188 / 171, 290 / 298; 12 of 64 in float 165 / 171, 261 / 290.  Four / one, forward, 36 of 64 in bfloat16 x 1024 50 / 56;
    // backward, 18 heads 87 / 97.
    const int vw = 16 * (w.terms == 1 ? kRowGroups<1> : kRowGroups<3>);
    const int64_t blocks = (int64_t)p->B * p->Hv * ((p->Dv + vw - 1) / vw) * (backward ? 2 : 1);
    int64_t segs = sm_count() / blocks;
    if (segs > w.chunks / 4) segs = w.chunks / 4;
    if (segs < 3 || (segs == 3 && !backward && w.chunks <= 32)) segs = 1;
    w.seg_chunks = (int)((w.chunks + segs - 1) / segs);
    w.segs = w.chunks > 0 ? (w.chunks + w.seg_chunks - 1) / w.seg_chunks : 1;
    // Room for as many segments as this call or any shorter or smaller one has over all its heads, so that a workspace
    // for the largest call serves them all: one block a segment at least, four chunks in each.
    int64_t most = (int64_t)p->B * p->Hv * (w.chunks / 4);
    if (most > sm_count() / (backward ? 2 : 1)) most = sm_count() / (backward ? 2 : 1);
    if (w.chunks / 4 >= 3) {
        w.seg_state = part((double)most * p->Dv * p->Dk * 4);
        w.seg_map = part((double)most * p->Dk * p->Dk * 4);
    }
    const size_t nc = (size_t)p->B * p->Hv * w.chunks, rows = (size_t)p->B * p->L;
    if (w.terms == 3) {
        w.q = part((double)rows * p->Hk * p->Dk * 6);
        w.k = w.q;
        w.v = part((double)rows * p->Hv * p->Dv * 6);
        w.go = backward ? w.v : 0;
    }
    w.coef = part((double)nc * kCoef * kC * 4);
    w.tri = part((double)nc * nt * kTri * 2);
    w.p = w.tri;
    if (backward) {
        const double nv = (double)nc * w.vblocks;
        w.r = part(nv * kTile * 4);
        w.s0 = part(nv * kC * w.dk * 4);
        w.rbt = w.terms == 3 ? w.v : part((double)rows * p->Hv * p->Dv * 2);     // bfloat16: the first of two terms is dV
    }
    w.total = w.q + w.k + w.v + w.go + w.coef + w.tri + w.p + 2 * (w.r + w.s0) + w.rbt + (backward ? 4 : 2) * w.seg_state + w.seg_map;
    return w;
}

// Chunk kernels number chunks of heads in one grid dimension.
bool chunks_fit(const cawn_delta_params *p) { return (double)p->B * p->Hv * ((double)p->L / kC + 1.0) < 2147483647.0; }

struct Carver {
    char *at;
    template <class T> T *take(size_t bytes)
    {
        T *p = reinterpret_cast<T *>(at);
        at += bytes;
        return p;
    }
};

// One sequence array as bfloat16 terms: itself, or (float storage) to be split into the workspace.
Terms terms_of(SplitJobs &jobs, const void *src, long long stride, const cawn_delta_params *p, int width, const Plan &w, size_t bytes, Carver &ws)
{
    if (w.terms == 1) return {static_cast<const bf16 *>(src), 0, stride, stride * p->L};
    bf16 *dst = ws.take<bf16>(bytes);
    jobs.job[jobs.count++] = {static_cast<const float *>(src), dst, stride, width};
    return {dst, jobs.rows * width, width, (long long)width * p->L};
}

// The shared part of both directions' arguments; grad_o NULL in the forward.
int chunk_params(ChunkParams &C, const cawn_delta_params *p, const DeltaParams &D, const Plan &w, const void *grad_o, Carver &ws, cudaStream_t st)
{
    C.g = D.g; C.beta = D.beta; C.state_in = D.state_in;
    C.L = p->L; C.B = p->B; C.Hk = p->Hk; C.Hv = p->Hv; C.Dk = p->Dk; C.Dv = p->Dv; C.scale = p->scale;
    C.chunks = w.chunks; C.vblocks = w.vblocks; C.segs = w.segs; C.seg_chunks = w.seg_chunks;
    SplitJobs jobs = {};
    jobs.rows = (long long)p->B * p->L;
    C.q = terms_of(jobs, D.q, D.q_stride, p, p->Hk * p->Dk, w, w.q, ws);
    C.k = terms_of(jobs, D.k, D.k_stride, p, p->Hk * p->Dk, w, w.k, ws);
    C.v = terms_of(jobs, D.v, D.v_stride, p, p->Hv * p->Dv, w, w.v, ws);
    if (grad_o != nullptr) C.go = terms_of(jobs, grad_o, D.o_stride, p, p->Hv * p->Dv, w, w.go, ws);
    C.coef = ws.take<float>(w.coef);
    C.tri = ws.take<bf16>(w.tri);
    C.p = ws.take<bf16>(w.p);
    C.seg_start = ws.take<float>(w.seg_state);
    C.seg_end = ws.take<float>(w.seg_state);
    C.seg_map = ws.take<float>(w.seg_map);
    return jobs.count == 0 ? CAWN_OK : status_of(launch_delta_split(jobs, st));
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
    if (!chunks_fit(params)) return CAWN_ERR_UNSUPPORTED;
    *bytes = params->L == 0 ? 0 : plan_of(params, op == CAWN_DELTA_BWD).total;
    return CAWN_OK;
}

extern "C" int cawn_delta_rule_fwd(const cawn_delta_params *params, const void *q, const void *k, const void *v, const float *g,
                                   const float *beta, const float *state_in, void *o, float *state_out, void *workspace,
                                   size_t workspace_bytes, void *cuda_stream)
{
    using namespace cawn;
    int rc = check(params);
    if (rc != CAWN_OK) return rc;
    if (params->L <= step_tokens(params)) return cawn_delta_rule_step(params, q, k, v, g, beta, state_in, o, state_out, cuda_stream);
    if (!chunks_fit(params)) return CAWN_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (q == nullptr || k == nullptr || v == nullptr || g == nullptr || beta == nullptr || o == nullptr || workspace == nullptr)
        return CAWN_ERR_NULL_POINTER;
    if (!all_aligned16(q, k, v, g, beta, state_in, o, state_out, workspace)) return CAWN_ERR_MISALIGNED;
    const Plan w = plan_of(params, false);
    if (workspace_bytes < w.total) return CAWN_ERR_WORKSPACE_TOO_SMALL;
    const DeltaParams D = fill(params, q, k, v, g, beta, state_in);
    ChunkParams C = {};
    Carver ws = {static_cast<char *>(workspace)};
    rc = chunk_params(C, params, D, w, nullptr, ws, st);
    if (rc != CAWN_OK) return rc;
    C.o = o; C.state_out = state_out; C.o_stride_t = D.o_stride; C.o_stride_b = D.o_stride * params->L;
    cudaError_t e = launch_delta_prep(C, w.dk, w.terms, st);
    if (e == cudaSuccess) e = launch_delta_scan(C, w.dk, w.terms, st);
    return status_of(e);
}

extern "C" int cawn_delta_rule_bwd(const cawn_delta_params *params, const void *q, const void *k, const void *v, const float *g,
                                   const float *beta, const float *state_in, const void *grad_o, const float *grad_state_out,
                                   void *grad_q, void *grad_k, void *grad_v, float *grad_g, float *grad_beta, float *grad_state_in,
                                   void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    using namespace cawn;
    int rc = check(params);
    if (rc != CAWN_OK) return rc;
    if (!chunks_fit(params)) return CAWN_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (!all_aligned16(q, k, v, g, beta, state_in, grad_o, grad_state_out, grad_q, grad_k, grad_v, grad_g, grad_beta, grad_state_in, workspace))
        return CAWN_ERR_MISALIGNED;
    if (params->L == 0) return pass_state(params, grad_state_out, grad_state_in, st);
    if (q == nullptr || k == nullptr || v == nullptr || g == nullptr || beta == nullptr || grad_o == nullptr || grad_q == nullptr ||
        grad_k == nullptr || grad_v == nullptr || grad_g == nullptr || grad_beta == nullptr || workspace == nullptr)
        return CAWN_ERR_NULL_POINTER;
    const Plan w = plan_of(params, true);
    if (workspace_bytes < w.total) return CAWN_ERR_WORKSPACE_TOO_SMALL;
    const DeltaParams D = fill(params, q, k, v, g, beta, state_in);
    ChunkParams C = {};
    Carver ws = {static_cast<char *>(workspace)};
    rc = chunk_params(C, params, D, w, grad_o, ws, st);
    if (rc != CAWN_OK) return rc;
    C.adj_start = ws.take<float>(w.seg_state);
    C.adj_end = ws.take<float>(w.seg_state);
    C.adj_in = grad_state_out; C.adj_out = grad_state_in;
    C.r = ws.take<float>(w.r);
    C.dk = ws.take<float>(w.r);
    C.s0 = ws.take<float>(w.s0);
    C.ds = ws.take<float>(w.s0);
    C.rbt = ws.take<bf16>(w.rbt);
    C.o = grad_v;
    const long long vo = (long long)params->Hv * params->Dv;
    C.rb = {nullptr, (long long)params->B * params->L * vo, vo, vo * params->L};
    C.gq = grad_q; C.gk = grad_k; C.gg = grad_g; C.gbeta = grad_beta;
    cudaError_t e = launch_delta_prep(C, w.dk, w.terms, st);
    if (e == cudaSuccess && w.segs > 1) {
        e = launch_delta_walks(C, w.dk, w.terms, true, st);
        if (e == cudaSuccess) e = launch_delta_join(C, w.dk, true, st);
    }
    if (e == cudaSuccess) e = launch_delta_walks(C, w.dk, w.terms, false, st);
    if (e == cudaSuccess) e = launch_delta_grads(C, w.dk, w.terms, st);
    return status_of(e);
}
