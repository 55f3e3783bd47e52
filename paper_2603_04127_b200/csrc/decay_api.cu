// Host side of attention with a decay per head: descriptor validation, plan object, the passes of a call.
#include "decay.cuh"

#include <math.h>
#include <new>

namespace darkattn {

static bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
template <typename... P> static bool all_set(const P *...p) { return ((p != nullptr) && ...); }
template <typename... P> static bool all_aligned(const P *...p) { return (aligned16(p) && ...); }
static bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// bytes of the arrays of a call
struct Sizes {
    size_t q, k, v, o, s, g, n;
    explicit Sizes(const darkattn_decay_desc_t &ds)
    {
        const size_t e = ds.dtype == DARKATTN_BF16 ? 2 : 4, rows = (size_t)ds.B * ds.N * e;
        q = rows * ds.H * ds.d; k = rows * ds.H_kv * ds.d; v = rows * ds.H_kv * ds.dv; o = rows * ds.H * ds.dv;
        s = (size_t)ds.B * ds.H_kv * ds.d * ds.dv * 4; g = (size_t)ds.H_kv * 4; n = (size_t)ds.B * 4;
    }
};

static DecayArgs common_args(const darkattn_decay_plan_s *plan, const float *log_decay, const int *lengths, int nseg, int cps, int sub, void *ws)
{
    DecayArgs A = {};
    A.log_decay = log_decay;
    A.lengths = lengths;
    A.B = plan->desc.B; A.Hkv = plan->desc.H_kv; A.N = plan->desc.N;
    A.nseg = nseg; A.cps = cps; A.sub = sub;
    A.status = static_cast<int *>(ws);
    return A;
}

static darkattn_status_t run(const darkattn_decay_plan_s *plan, DecayArgs &A, DecayPass *states, int nstate, cudaStream_t st)
{
    if (plan->path == DARKATTN_PATH_TENSOR) return decay_tc_run(A, states, nstate, st);
    return decay_simt_run(A, states, nstate, plan->desc.dtype == DARKATTN_BF16, st);
}

}  // namespace darkattn

using namespace darkattn;

extern "C" {

darkattn_status_t darkattn_decay_plan(const darkattn_decay_desc_t *desc, darkattn_decay_plan_t *out)
{
    if (!desc || !out) return DARKATTN_ERR_INVALID_ARG;
    *out = nullptr;
    darkattn_decay_desc_t ds = *desc;
    if (ds.B < 1 || ds.H < 1 || ds.N < 1 || ds.d < 1 || ds.dv < 0 || ds.H_kv < 0) return DARKATTN_ERR_INVALID_ARG;
    if (ds.H_kv == 0) ds.H_kv = ds.H;
    if (ds.H_kv > ds.H || ds.H % ds.H_kv) return DARKATTN_ERR_INVALID_ARG;
    if (ds.dtype != DARKATTN_F32 && ds.dtype != DARKATTN_BF16) return DARKATTN_ERR_INVALID_ARG;
    if (ds.path < DARKATTN_PATH_AUTO || ds.path > DARKATTN_PATH_TENSOR) return DARKATTN_ERR_INVALID_ARG;
    if (!(ds.scale >= 0.f) || !isfinite(ds.scale)) return DARKATTN_ERR_INVALID_ARG;
    if (ds.dv == 0) ds.dv = ds.d;
    if (ds.scale == 0.f) ds.scale = 1.0f / sqrtf((float)ds.d);
    if ((long long)ds.B * ds.H > 65535 || ds.d > 512 || ds.dv > 512 || ds.N > (1 << 30)) return DARKATTN_ERR_UNSUPPORTED;
    const bool tensor_ok = decay_tc_supported(ds);
    if (ds.path == DARKATTN_PATH_TENSOR && !tensor_ok) return DARKATTN_ERR_UNSUPPORTED;

    darkattn_decay_plan_s *p = new (std::nothrow) darkattn_decay_plan_s();
    if (!p) return DARKATTN_ERR_INVALID_ARG;
    p->desc = ds;
    p->path = ds.path == DARKATTN_PATH_AUTO ? (tensor_ok ? DARKATTN_PATH_TENSOR : DARKATTN_PATH_SIMT) : ds.path;
    if (p->path == DARKATTN_PATH_TENSOR) decay_tc_split(p);
    else decay_simt_split(p);
    // states of the pieces: one set forwards, for a backward pass one more
    const size_t set = (size_t)ds.B * ds.H_kv * ds.d * ds.dv * sizeof(float);
    const size_t nf = set * ((p->fwd.nseg - 1) * p->fwd.sub), nb = set * ((p->bwd.nseg - 1) * p->bwd.sub);
    p->ws.status = 0;
    p->ws.seg[0] = 256;
    p->ws.seg[1] = 256 + ((nb + 255) & ~(size_t)255);
    const size_t fwd = 256 + nf, bwd = p->ws.seg[1] + nb;
    p->workspace_bytes = ((fwd > bwd ? fwd : bwd) + 255) & ~(size_t)255;
    *out = p;
    return DARKATTN_OK;
}

size_t darkattn_decay_workspace_bytes(darkattn_decay_plan_t plan) { return plan ? plan->workspace_bytes : 0; }
int32_t darkattn_decay_plan_path(darkattn_decay_plan_t plan) { return plan ? plan->path : -1; }
void darkattn_decay_destroy(darkattn_decay_plan_t plan) { delete plan; }

darkattn_status_t darkattn_decay_forward(darkattn_decay_plan_t plan, const void *Q, const void *K, const void *V, const float *log_decay,
                                         const int32_t *lengths, const float *S_in, void *O, float *S_out, void *workspace, void *cuda_stream)
{
    if (!plan || !all_set(Q, K, V, O) || !log_decay) return DARKATTN_ERR_INVALID_ARG;
    if (!workspace) return DARKATTN_ERR_WORKSPACE;
    if (!all_aligned(Q, K, V, O, workspace) || !all_aligned(S_in, S_out) || !aligned4(log_decay) || !aligned4(lengths)) return DARKATTN_ERR_INVALID_ARG;
    const darkattn_decay_desc_t &ds = plan->desc;
    const Sizes z(ds);
    if (clash({{O, z.o}, {S_out, z.s}, {workspace, plan->workspace_bytes}}, {{Q, z.q}, {K, z.k}, {V, z.v}, {log_decay, z.g}, {lengths, z.n}, {S_in, z.s}})) return DARKATTN_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    DecayArgs A = common_args(plan, log_decay, lengths, plan->fwd.nseg, plan->fwd.cps, plan->fwd.sub, workspace);
    float *seg = reinterpret_cast<float *>(static_cast<char *>(workspace) + plan->ws.seg[0]);
    A.npass = 1;
    A.pass[0] = DecayPass{Q, K, V, O, S_in, S_out, seg, ds.d, ds.dv, ds.H, ds.H_kv, 0, 0, ds.scale, ds.scale, 1.f, S_out != nullptr};
    DecayPass states = A.pass[0];
    return run(plan, A, &states, 1, st);
}

darkattn_status_t darkattn_decay_backward(darkattn_decay_plan_t plan, const void *Q, const void *K, const void *V, const float *log_decay,
                                          const int32_t *lengths, const float *S_in, const void *dO, const float *dS_out, void *dQ, void *dK, void *dV,
                                          float *dS_in, void *workspace, void *cuda_stream)
{
    if (!plan || !all_set(Q, K, V, dO, dQ, dK, dV) || !log_decay) return DARKATTN_ERR_INVALID_ARG;
    if (!workspace) return DARKATTN_ERR_WORKSPACE;
    if (!all_aligned(Q, K, V, dO, dQ, dK, dV, workspace) || !all_aligned(S_in, dS_out, dS_in) || !aligned4(log_decay) || !aligned4(lengths)) return DARKATTN_ERR_INVALID_ARG;
    const darkattn_decay_desc_t &ds = plan->desc;
    const Sizes z(ds);
    if (clash({{dQ, z.q}, {dK, z.k}, {dV, z.v}, {dS_in, z.s}, {workspace, plan->workspace_bytes}},
              {{Q, z.q}, {K, z.k}, {V, z.v}, {log_decay, z.g}, {lengths, z.n}, {S_in, z.s}, {dO, z.o}, {dS_out, z.s}})) return DARKATTN_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    DecayArgs A = common_args(plan, log_decay, lengths, plan->bwd.nseg, plan->bwd.cps, plan->bwd.sub, workspace);
    float *S = reinterpret_cast<float *>(static_cast<char *>(workspace) + plan->ws.seg[0]), *R = reinterpret_cast<float *>(static_cast<char *>(workspace) + plan->ws.seg[1]);
    A.npass = 3;
    A.pass[0] = DecayPass{dO, V, K, dQ, S_in, nullptr, S, ds.dv, ds.d, ds.H, ds.H_kv, 0, 1, ds.scale, ds.scale, 1.f, 0};
    A.pass[1] = DecayPass{V, dO, Q, dK, dS_out, nullptr, R, ds.dv, ds.d, ds.H_kv, ds.H, 1, 1, ds.scale, 1.f, ds.scale, 0};
    A.pass[2] = DecayPass{K, Q, dO, dV, dS_out, dS_in, R, ds.d, ds.dv, ds.H_kv, ds.H, 1, 0, ds.scale, 1.f, ds.scale, dS_in != nullptr};
    DecayPass sets[2] = {{nullptr, K, V, nullptr, S_in, nullptr, S, ds.d, ds.dv, ds.H_kv, ds.H_kv, 0, 0, 0.f, 0.f, 1.f, 0}, A.pass[2]};
    A.zero = lengths != nullptr;
    return run(plan, A, sets, 2, st);
}

darkattn_status_t darkattn_decay_step(darkattn_decay_plan_t plan, const void *q, const void *k, const void *v, const float *log_decay, float *S,
                                      const int32_t *slots, int32_t n_slots, void *o, void *cuda_stream)
{
    if (!plan || !all_set(q, k, v, o) || !log_decay || !S) return DARKATTN_ERR_INVALID_ARG;
    if (!all_aligned(q, k, v, o) || !aligned16(S) || !aligned4(log_decay) || !aligned4(slots)) return DARKATTN_ERR_INVALID_ARG;
    if (n_slots < 1 || (!slots && n_slots < plan->desc.B)) return DARKATTN_ERR_INVALID_ARG;
    return decay_step(plan, q, k, v, log_decay, S, slots, n_slots, o, static_cast<cudaStream_t>(cuda_stream));
}

darkattn_status_t darkattn_decay_last_device_status(darkattn_decay_plan_t plan, const void *workspace, void *cuda_stream)
{
    if (!plan || !workspace) return DARKATTN_ERR_INVALID_ARG;
    int word = 0;
    DARKATTN_CUDA_TRY(cudaStreamSynchronize(static_cast<cudaStream_t>(cuda_stream)), "decay_last_device_status: sync");
    DARKATTN_CUDA_TRY(cudaMemcpy(&word, workspace, sizeof(int), cudaMemcpyDeviceToHost), "decay_last_device_status: read");
    return word == 0 ? DARKATTN_OK : DARKATTN_ERR_TIMEOUT;
}

}  // extern "C"
