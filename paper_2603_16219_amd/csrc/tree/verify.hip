// The verify-and-recover step down a tree of drafts, for MI355X (gfx950); include/specsteer_tree.h says what it computes.
//
// A workgroup a sequence walks from the root: the sums of the cursor's rows of G and S_noctx, Eq. 7 on all children of the cursor at once, the first
// one accepted is the next cursor.  Where none is, or there are none, Eq. 8's row is drawn from by inverse CDF.
#include "../loss/loss_rows.h"
#include "tree_common.h"

namespace {

constexpr int kVerifyThreads = 512;

struct VerifyArgs {
    const void *G, *Sp, *Sm;
    const int32_t *tokens, *parents, *tree_len;
    const float* uniforms;
    int32_t *accepted_len, *path, *next_token;
    float* next_logprob;
    long sb, st;
    int N, V;
    Factor c;
    double c64, inv_tau, lambda, beta;
    int far, greedy, plain;  // plain: beta is 0
};

// the steering term's difference: a token that both of the specialist's rows mask has none
__device__ __forceinline__ double steer(float sp, float sm) { return sp == sm ? 0.0 : (double)sp - (double)sm; }

template <int DT>
__device__ __forceinline__ Total<Sum> sum_row(const VerifyArgs& a, const void* h, Total<Sum>* part, bool& far) {
    const Layout<DT> lay(h, a.V, threadIdx.x);
    const Sum mine = lane_sum<DT, Sum, 2>(h, nullptr, lay, threadIdx.x, lay.vecs, kVerifyThreads, true, a.c);
    Total<Sum> s = block_total(mine, kVerifyThreads, part);
    __syncthreads();
    far = a.far || is_far(s);
    if (far) s = far_sum<DT, Sum>(h, nullptr, a.V, a.c64, kVerifyThreads, part);
    return s;
}
// log2 of the row's sum of exponentials
__device__ __forceinline__ double log2_sum(const VerifyArgs& a, const Total<Sum>& s, bool far) {
    return (far ? (double)s.E * a.c64 : (double)s.E) + log2(s.s);
}

__device__ __forceinline__ int block_min(int v, int* part) {
    v = -wave_max_i32(-v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 0; w < kVerifyThreads / kWave; ++w) v = min(v, part[w]);
    return v;
}

template <int DT>
__global__ __launch_bounds__(kVerifyThreads) void verify_kernel(const VerifyArgs a) {
    constexpr int NT = kVerifyThreads, kWaves = NT / kWave;
    __shared__ Total<Sum> part[kWaves];
    __shared__ int ints[kWaves];
    __shared__ double sums[kWaves];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int N = a.tree_len ? a.tree_len[b] : a.N;
    const int32_t *y = a.tokens + (long)b * a.N, *up = a.parents ? a.parents + (long)b * a.N : nullptr;
    bool bad = N < 0 || N > a.N;
    if (!bad)
        for (int i = tid; i < N; i += NT) {
            const int p = up ? up[i] : i - 1;
            bad = bad || p < -1 || p >= i || y[i] < 0 || y[i] >= a.V;
        }
    bad = block_min(bad ? 0 : 1, ints) == 0;
    for (int i = tid; i < a.N; i += NT) a.path[(long)b * a.N + i] = -1;
    if (bad) {
        if (tid == 0) {
            a.accepted_len[b] = a.next_token[b] = -1;
            if (a.next_logprob) a.next_logprob[b] = __builtin_nanf("");
        }
        return;
    }
    int cur = -1, n = 0;
    for (;;) {
        const int none = 1 << 30;
        int child = none;
        for (int i = cur + 1 + tid; i < N; i += NT)
            if ((up ? up[i] : i - 1) == cur) child = min(child, i);
        if (block_min(child, ints) == none) break;
        const long at = b * a.sb + (cur + 1) * a.st;
        const void *g = row_ptr<DT>(a.G, at), *m = row_ptr<DT>(a.Sm, at);
        bool far_g, far_m;
        const Total<Sum> sg = sum_row<DT>(a, g, part, far_g), sm = sum_row<DT>(a, m, part, far_m);
        const double lg = log2_sum(a, sg, far_g), lm = log2_sum(a, sm, far_m);
        child = none;
        for (int i = cur + 1 + tid; i < N; i += NT)
            if ((up ? up[i] : i - 1) == cur) {
                const double hg = ld_elem<DT>(g, y[i]), hm = ld_elem<DT>(m, y[i]), u = a.uniforms[(long)b * (a.N + 1) + i];
                // masked by G: never accepted; by S_noctx alone: always
                const double alpha = hg == -__builtin_huge_val() ? -1.0 : exp2((hg * a.c64 - lg) - (hm * a.c64 - lm)) / a.lambda;
                if (u <= 1.0 && !(u > alpha)) child = min(child, i);
            }
        child = block_min(child, ints);
        if (child == none) break;
        if (tid == 0) a.path[(long)b * a.N + n] = child;
        ++n;
        cur = child;
    }
    const long at = b * a.sb + (cur + 1) * a.st;
    const void *g = row_ptr<DT>(a.G, at), *sp = row_ptr<DT>(a.Sp, at), *sm = row_ptr<DT>(a.Sm, at);
    // the mode first: the reference of the sums, and greedy decoding's token
    const auto rec = [&](int i) {
        const double h = ld_elem<DT>(g, i);
        return a.plain ? h : __dadd_rn(h, __dmul_rn(a.beta, steer(ld_elem<DT>(sp, i), ld_elem<DT>(sm, i))));
    };
    double top = -__builtin_huge_val();
    int mode = 1 << 30;
    for (int i = tid; i < a.V; i += NT) {
        const double h = rec(i);
        if (h > top) {
            top = h;
            mode = i;
        }
    }
    for (int d = 1; d < kWave; d <<= 1) {
        const double o = __shfl_xor(top, d, kWave);
        const int i = __shfl_xor(mode, d, kWave);
        if (o > top || (o == top && i < mode)) {
            top = o;
            mode = i;
        }
    }
    __syncthreads();
    if (lane == 0) {
        sums[wave] = top;
        ints[wave] = mode;
    }
    __syncthreads();
    for (int w = 0; w < kWaves; ++w)
        if (sums[w] > top || (sums[w] == top && ints[w] < mode)) {
            top = sums[w];
            mode = ints[w];
        }
    __syncthreads();
    const auto term = [&](int i) { return (double)exp2_hw((float)((rec(i) - top) * a.c64)); };
    double mine = 0.0;
    for (int i = tid; i < a.V; i += NT) mine += term(i);
    const auto all = [&](double v) {
        v = wave_sum_f64(v);
        __syncthreads();
        if (lane == 0) sums[wave] = v;
        __syncthreads();
        return wave_sum_f64(lane < kWaves ? sums[lane] : 0.0);
    };
    const double Z = all(mine), target = (double)a.uniforms[(long)b * (a.N + 1) + a.N] * Z;
    int token = min(mode, a.V - 1);
    if (!a.greedy) {
        double before = 0.0;
        int last = token;  // with any mass
        token = -1;
        for (int first = 0; first < a.V && token < 0; first += NT) {
            const int i = first + tid;
            const double t = i < a.V ? term(i) : 0.0, incl = wave_incl_scan_f64(t);
            __syncthreads();
            if (lane == 63) sums[wave] = incl;
            __syncthreads();
            double start = before;
            for (int w = 0; w < kWaves; ++w) {
                if (w < wave) start += sums[w];
                before += sums[w];
            }
            const int hit = block_min(t > 0.0 && start + incl > target ? i : 1 << 30, ints);
            if (hit < 1 << 30) token = hit;
            const int some = -block_min(t > 0.0 ? -i : 1, ints);
            if (some >= 0) last = some;
        }
        if (token < 0) token = last;
    }
    if (tid == 0) {
        a.accepted_len[b] = n;
        a.next_token[b] = token;
        if (a.next_logprob) a.next_logprob[b] = (float)((rec(token) - top) * a.inv_tau - log(Z));
    }
}

}  // namespace

extern "C" {

size_t specsteer_tree_verify_workspace_bytes(const ss_params* params) {
    long st, sb;
    return verify_shape(params, st, sb) == SS_OK ? 256 : 0;
}

ss_status specsteer_tree_verify(const void* G, const void* S_ctx, const void* S_noctx, const int32_t* tokens, const int32_t* parents,
                                const int32_t* tree_len, const float* uniforms, const ss_params* params, int32_t* accepted_len, int32_t* path,
                                int32_t* next_token, float* next_token_logprob, void* workspace, size_t workspace_bytes, void* stream) {
    long st, sb;
    const ss_status chk = verify_shape(params, st, sb);
    if (chk != SS_OK) return chk;
    if (params->batch == 0) return SS_OK;
    const bool nodes = params->k_max > 0;
    if (!G || !S_ctx || !S_noctx || !uniforms || !accepted_len || !next_token || (nodes && (!tokens || !path))) return SS_ERR_NULL;
    const uintptr_t elem = params->dtype == SS_BF16 ? 1 : 3;
    if ((reinterpret_cast<uintptr_t>(G) | reinterpret_cast<uintptr_t>(S_ctx) | reinterpret_cast<uintptr_t>(S_noctx)) & elem) return SS_ERR_STRIDE;
    if (bad_workspace(workspace, workspace_bytes, 256)) return SS_ERR_WORKSPACE;
    ss_loss_params lp{params->batch, params->k_max + 1, params->vocab, params->dtype, 0, 0, 0, 0, params->temperature, 1.f};
    const Rows r = make_rows(G, nullptr, nullptr, tokens, nullptr, lp, LossShape{});
    const VerifyArgs a{G, S_ctx, S_noctx, tokens, nodes ? parents : nullptr, tree_len, uniforms, accepted_len, path, next_token, next_token_logprob, sb, st,
                       params->k_max, params->vocab, r.c, r.c64, r.inv_tau, (double)params->lambda, (double)params->beta, r.far,
                       (params->flags & SS_FLAG_GREEDY) ? 1 : 0, params->beta == 0.f ? 1 : 0};
    launch(params->dtype == SS_BF16 ? verify_kernel<SS_BF16> : verify_kernel<SS_F32>, dim3((unsigned)params->batch), dim3(kVerifyThreads), 0,
           static_cast<hipStream_t>(stream), a);
    return tree_launched();
}

}  // extern "C"
