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

// (lse in log2 units, D = sum(out dout)) of every query row, 8 columns per lane:
// what the backward's kernels read of a row beside q and dout.  Bound by the
// rows of out and dout, which it reads once.
template <typename ST, int DH>
__global__ __launch_bounds__(256) void wattn_ld_kernel(AttnArgs a, uint32_t first) {
    constexpr int L = DH / 8;
    const int64_t row = ((int64_t)first + blockIdx.x) * (256 / L) + threadIdx.x / L;
    if (row >= (int64_t)a.B * a.Hq * a.Tq) return;
    const int li = threadIdx.x % L;
    const int i = (int)(row % a.Tq), h = (int)(row / a.Tq % a.Hq), b = (int)(row / a.Tq / a.Hq);
    float d = 0.f;
    const bool live = i < seq_len_of(a.ql, b, a.Tq);
    if (live) {
        float x[8], y[8];
        frag8_to_f32<ST>(frag8_load<ST>(row_ptr<ST>(a.out, b, h, i) + 8 * li), x);
        frag8_to_f32<ST>(frag8_load<ST>(row_ptr<ST>(a.dout, b, h, i) + 8 * li), y);
#pragma unroll
        for (int e = 0; e < 8; ++e) d += x[e] * y[e];
    }
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) d += __shfl_xor(d, o, 64);
    if (li == 0) {
        const float l = live ? a.lse[row] : -__builtin_inff();
        a.ld[row] = make_float2(l == -__builtin_inff() ? __builtin_inff() : l * kLog2e, d);
    }
}

// One wave per query row, and one per key row.
template <typename ST, int DH>
__global__ __launch_bounds__(256) void wattn_dq_rows_kernel(AttnArgs a, uint32_t first) {
    const int lane = threadIdx.x & 63;
    const int64_t row = ((int64_t)first + blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)a.B * a.Hq * a.Tq) return;
    const int i = (int)(row % a.Tq), h = (int)(row / a.Tq % a.Hq), b = (int)(row / a.Tq / a.Hq);
    const int qn = seq_len_of(a.ql, b, a.Tq), kn = seq_len_of(a.kl, b, a.N);
    const float zero[RowLanes<DH>::N] = {};
    if (i < qn) row_dq<ST, DH>(a, b, h, i, kn - qn + i, kn, lane);
    else row_store<ST, DH>(row_ptr<ST>(a.dq, b, h, i), lane, zero, 0.f);
}

template <typename ST, int DH>
__global__ __launch_bounds__(256) void wattn_dkv_rows_kernel(AttnArgs a, uint32_t first) {
    const int lane = threadIdx.x & 63;
    const int64_t row = ((int64_t)first + blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)a.B * a.Hkv * a.N) return;
    const int j = (int)(row % a.N), hk = (int)(row / a.N % a.Hkv), b = (int)(row / a.N / a.Hkv);
    const int qn = seq_len_of(a.ql, b, a.Tq), kn = seq_len_of(a.kl, b, a.N), off = kn - qn;
    float dk[RowLanes<DH>::N] = {}, dv[RowLanes<DH>::N] = {};
    if (j < kn)
        row_dkv<ST, DH>(a, b, hk, j, off, min(max(0, j - off), qn) * a.G, qn * a.G, [&](int p) { return sees(a, p, j); }, lane, dk,
                        dv);
    row_store<ST, DH>(row_ptr<ST>(a.dk, b, hk, j), lane, dk, 1.f);
    row_store<ST, DH>(row_ptr<ST>(a.dv, b, hk, j), lane, dv, 1.f);
}

template <class K>
int launch_rows(K kern, int64_t rows, int per_block, const AttnArgs& a, hipStream_t stream) {
    return launch_parts((uint64_t)(rows + per_block - 1) / per_block, 256, [&](uint32_t first, uint32_t blocks) {
        hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), 0, stream, a, first);
        return hipGetLastError() == hipSuccess ? 0 : -1;
    });
}

size_t ld_bytes(const AttnArgs& a) { return ((size_t)a.B * a.Hq * a.Tq * sizeof(float2) + 255) / 256 * 256; }

}  // namespace

size_t attn_fwd_scratch(int dtype, int dh, const AttnArgs& a) {
    return dtype == kBF16 ? wattn_tiled_scratch(dh, a) : 0;
}
size_t attn_bwd_scratch(int dtype, int dh, const AttnArgs& a) {
    return ld_bytes(a) + (dtype == kBF16 ? wattn_bwd_sums(dh, a) : 0);
}

int launch_window_attn(int dtype, int dh, const AttnArgs& a, float* part, hipStream_t stream) {
    if (dtype == kBF16) return launch_wattn_tiled(dh, a, part, stream);
    return heads_by_type(dtype, dh, [&](auto st, auto d) {
        return launch_rows(wattn_rows_kernel<decltype(st), decltype(d)::value>, (int64_t)a.B * a.Hq * a.Tq, 4, a, stream);
    });
}

int launch_window_attn_bwd(int dtype, int dh, AttnArgs a, void* scratch, hipStream_t stream) {
    a.ld = static_cast<float2*>(scratch);
    const int64_t qrows = (int64_t)a.B * a.Hq * a.Tq, krows = (int64_t)a.B * a.Hkv * a.N;
    return heads_by_type(dtype, dh, [&](auto st, auto d) {
        using ST = decltype(st);
        constexpr int DH = decltype(d)::value;
        int e = launch_rows(wattn_ld_kernel<ST, DH>, qrows, 256 / (DH / 8), a, stream);
        if (e) return e;
        if (dtype == kBF16)
            return launch_wattn_bwd_tiled(dh, a, reinterpret_cast<float*>(static_cast<char*>(scratch) + ld_bytes(a)), stream);
        e = launch_rows(wattn_dq_rows_kernel<ST, DH>, qrows, 4, a, stream);
        return e ? e : launch_rows(wattn_dkv_rows_kernel<ST, DH>, krows, 4, a, stream);
    });
}

}  // namespace mosa
