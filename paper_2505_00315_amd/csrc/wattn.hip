// Causal attention with a sliding window and first tokens that stay visible.
#include "heads.h"
#include "launch_parts.h"
#include "rowattn.h"

namespace mosa {

namespace {

template <typename ST, int DH>
__device__ __forceinline__ void row_store(ST* p, int lane, const float (&x)[RowLanes<DH>::N], float f) {
#pragma unroll
    for (int i = 0; i < RowLanes<DH>::N; ++i)
        if (RowLanes<DH>::has(lane)) st1<ST>(p + lane + 64 * i, x[i] * f);
}

// One wave per query row.
template <typename ST, int DH>
__global__ __launch_bounds__(256) void wattn_rows_kernel(AttnArgs a, uint32_t first) {
    const int lane = threadIdx.x & 63;
    const int64_t row = ((int64_t)first + blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)a.B * a.Hq * a.Tq) return;
    const int i = (int)(row % a.Tq), h = (int)(row / a.Tq % a.Hq), b = (int)(row / a.Tq / a.Hq);
    const int qn = seq_len_of(a.ql, b, a.Tq), kn = seq_len_of(a.kl, b, a.N), p = kn - qn + i;
    float q[RowLanes<DH>::N], o[RowLanes<DH>::N] = {}, m = -__builtin_inff(), l = 0.f;
    if (i < qn) {
        row_load<ST, DH>(row_ptr<ST>(a.q, b, h, i), lane, q);
        const KeyList list = keys_of(a, p, p, kn);
        row_attend<DH>(a, WideKeys<ST, DH>{a, b, h / a.G}, [&](int e) { return list.key(e); }, 0, list.count, p, kn, q,
                       lane, m, l, o);
    }
    row_finish<ST, DH>(a, b, h, i, row, lane, m, l, o, nullptr, nullptr);
}

// D = sum(out dout) of a query row (0 past the length).
template <typename ST, int DH>
__global__ __launch_bounds__(256) void wattn_d_kernel(AttnArgs a, uint32_t first) {
    const int lane = threadIdx.x & 63;
    const int64_t row = ((int64_t)first + blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)a.B * a.Hq * a.Tq) return;
    const int i = (int)(row % a.Tq), h = (int)(row / a.Tq % a.Hq), b = (int)(row / a.Tq / a.Hq);
    float x[RowLanes<DH>::N], y[RowLanes<DH>::N], d = 0.f;
    if (i < seq_len_of(a.ql, b, a.Tq)) {
        row_load<ST, DH>(row_ptr<ST>(a.out, b, h, i), lane, x);
        row_load<ST, DH>(row_ptr<ST>(a.dout, b, h, i), lane, y);
        d = row_dot<DH>(x, y);
    }
    if (lane == 0) a.D[row] = d;
}

// One wave per query row: dq = scale sum_j ds_j k_j, ds = p (dout v_j - D).
template <typename ST, int DH>
__global__ __launch_bounds__(256) void wattn_dq_rows_kernel(AttnArgs a, uint32_t first) {
    constexpr int N = RowLanes<DH>::N;
    const int lane = threadIdx.x & 63;
    const int64_t row = ((int64_t)first + blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)a.B * a.Hq * a.Tq) return;
    const int i = (int)(row % a.Tq), h = (int)(row / a.Tq % a.Hq), b = (int)(row / a.Tq / a.Hq);
    const int qn = seq_len_of(a.ql, b, a.Tq), kn = seq_len_of(a.kl, b, a.N), p = kn - qn + i;
    float dq[N] = {};
    if (i < qn) {
        float q[N], g[N], k[N], v[N];
        row_load<ST, DH>(row_ptr<ST>(a.q, b, h, i), lane, q);
        row_load<ST, DH>(row_ptr<ST>(a.dout, b, h, i), lane, g);
        const float lse = a.lse[row], D = a.D[row];
        const KeyList list = keys_of(a, p, p, kn);
        const WideKeys<ST, DH> keys{a, b, h / a.G};
        for (int e = 0; e < list.count; ++e) {
            keys.load(list.key(e), lane, k, v);
            const float w = __builtin_amdgcn_exp2f((row_dot<DH>(q, k) * a.scale - lse) * kLog2e);
            const float ds = w * (row_dot<DH>(g, v) - D) * a.scale;
#pragma unroll
            for (int n = 0; n < N; ++n) dq[n] += ds * k[n];
        }
    }
    row_store<ST, DH>(row_ptr<ST>(a.dq, b, h, i), lane, dq, 1.f);
}

// One wave per key row: dv = sum_i p_i dout_i, dk = scale sum_i ds_i q_i over
// the queries that see it, of every query head of the group.
template <typename ST, int DH>
__global__ __launch_bounds__(256) void wattn_dkv_rows_kernel(AttnArgs a, uint32_t first) {
    constexpr int N = RowLanes<DH>::N;
    const int lane = threadIdx.x & 63;
    const int64_t row = ((int64_t)first + blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)a.B * a.Hkv * a.N) return;
    const int j = (int)(row % a.N), hk = (int)(row / a.N % a.Hkv), b = (int)(row / a.N / a.Hkv);
    const int qn = seq_len_of(a.ql, b, a.Tq), kn = seq_len_of(a.kl, b, a.N), off = kn - qn;
    float dk[N] = {}, dv[N] = {};
    if (j < kn) {
        float q[N], g[N], k[N], v[N];
        const WideKeys<ST, DH> keys{a, b, hk};
        keys.load(j, lane, k, v);
        for (int h = hk * a.G; h < (hk + 1) * a.G; ++h)
            for (int i = max(0, j - off); i < qn; ++i) {
                if (!sees(a, off + i, j)) break;
                const int64_t qr = ((int64_t)b * a.Hq + h) * a.Tq + i;
                row_load<ST, DH>(row_ptr<ST>(a.q, b, h, i), lane, q);
                row_load<ST, DH>(row_ptr<ST>(a.dout, b, h, i), lane, g);
                const float w = __builtin_amdgcn_exp2f((row_dot<DH>(q, k) * a.scale - a.lse[qr]) * kLog2e);
                const float ds = w * (row_dot<DH>(g, v) - a.D[qr]) * a.scale;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    dk[n] += ds * q[n];
                    dv[n] += w * g[n];
                }
            }
    }
    row_store<ST, DH>(row_ptr<ST>(a.dk, b, hk, j), lane, dk, 1.f);
    row_store<ST, DH>(row_ptr<ST>(a.dv, b, hk, j), lane, dv, 1.f);
}

template <class K>
int launch_rows(K kern, int64_t rows, const AttnArgs& a, hipStream_t stream) {
    return launch_parts((uint64_t)(rows + 3) / 4, 256, [&](uint32_t first, uint32_t blocks) {
        hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), 0, stream, a, first);
        return hipGetLastError() == hipSuccess ? 0 : -1;
    });
}

template <typename ST, int DH>
int bwd_t(const AttnArgs& a, hipStream_t stream) {
    const int64_t qrows = (int64_t)a.B * a.Hq * a.Tq, krows = (int64_t)a.B * a.Hkv * a.N;
    int e = launch_rows(wattn_d_kernel<ST, DH>, qrows, a, stream);
    if (!e) e = launch_rows(wattn_dq_rows_kernel<ST, DH>, qrows, a, stream);
    if (!e) e = launch_rows(wattn_dkv_rows_kernel<ST, DH>, krows, a, stream);
    return e;
}

}  // namespace

size_t attn_fwd_scratch(int dtype, int dh, const AttnArgs& a) {
    return dtype == kBF16 ? wattn_tiled_scratch(dh, a) : 0;
}
size_t attn_bwd_scratch(const AttnArgs& a) { return (size_t)a.B * a.Hq * a.Tq * sizeof(float); }

int launch_window_attn(int dtype, int dh, const AttnArgs& a, float* part, hipStream_t stream) {
    if (dtype == kBF16) return launch_wattn_tiled(dh, a, part, stream);
    return heads_by_type(dtype, dh, [&](auto st, auto d) {
        return launch_rows(wattn_rows_kernel<decltype(st), decltype(d)::value>, (int64_t)a.B * a.Hq * a.Tq, a, stream);
    });
}

int launch_window_attn_bwd(int dtype, int dh, const AttnArgs& a, hipStream_t stream) {
    return heads_by_type(dtype, dh, [&](auto st, auto d) { return bwd_t<decltype(st), decltype(d)::value>(a, stream); });
}

}  // namespace mosa
