// Operators around a block (residual stream with norms, products with weight
// matrices, log probabilities of tokens): arguments shared by their kernels and
// the host layer.
#pragma once

#include "heads.h"

namespace mosa {

constexpr int kCus = 256;  // of the chip

// Sums of many terms whose result is stored.  With fp32 storage they are taken in
// 64 bits, so that the result is rounded once; with bf16 storage in fp32 by lane, in
// order, and in 64 bits from the workgroups' partials on.  A lane's terms are the rows
// over its workgroup's share: 32 of 16384 rows of 4096, 256 of 65536 rows of 8192, some
// 2^15 where the longest inputs fill a card.  n terms are off by at most n 2^-24 of the
// sum of their magnitudes, so by less than bf16's half step of 2^-8 of it even then.
template <typename ST>
using WideSum = std::conditional_t<sizeof(ST) == 4, double, float>;
inline size_t wide_sum_bytes(int dtype) { return dtype == kBF16 ? sizeof(float) : sizeof(double); }

// 16 bytes of a row: 8 bf16 or 4 fp32 values.
template <typename ST>
struct Unit {
    static constexpr int E = 16 / (int)sizeof(ST);
    uint4 u;
    __device__ __forceinline__ void get(float (&x)[E]) const {
        if constexpr (sizeof(ST) == 2) {
            Frag8<uint16_t> f;
            f.v = __builtin_bit_cast(bf16x8, u);
            frag8_to_f32<uint16_t>(f, x);
        } else {
            x[0] = __uint_as_float(u.x), x[1] = __uint_as_float(u.y), x[2] = __uint_as_float(u.z), x[3] = __uint_as_float(u.w);
        }
    }
    __device__ __forceinline__ void set(const float (&x)[E]) {
        if constexpr (sizeof(ST) == 2) u = __builtin_bit_cast(uint4, frag8_from<uint16_t>(x).v);
        else u = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    __device__ __forceinline__ void load(const ST* p) { u = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(ST* p) const { *reinterpret_cast<uint4*>(p) = u; }
};

// Partial sums [parts][n][cols] (WideSums) added in a fixed order, in 64 bits, into the
// out[i] that are not NULL, stored in `dtype`.
struct SumParts {
    const void* partial;
    int parts, n, cols;
    void* out[3];
};
int launch_sum_parts(int dtype, const SumParts& s, hipStream_t stream);
// Columns 32 block .. + 31 of vector `which`, by T lanes: T / 32 strands of parts, then the strands in order.
// red: T doubles of LDS.
template <typename ST, int T>
__device__ __forceinline__ void sum_parts_columns(const SumParts& s, int which, int block, double* red) {
    if (!s.out[which]) return;
    const WideSum<ST>* p = static_cast<const WideSum<ST>*>(s.partial) + (size_t)which * s.cols;
    const int c = threadIdx.x & 31, strand = threadIdx.x >> 5, col = block * 32 + c;
    double x = 0.0;
    if (col < s.cols) {
#pragma unroll 8
        for (int i = strand; i < s.parts; i += T / 32) x += p[(size_t)i * s.n * s.cols + col];
    }
    red[threadIdx.x] = x;
    __syncthreads();
    if (threadIdx.x < 32 && col < s.cols) {
        double t = 0.0;
        for (int i = 0; i < T / 32; ++i) t += red[32 * i + c];
        st1<ST>(static_cast<ST*>(s.out[which]) + col, (float)t);
    }
}

// ---------------------------------------------------------------------------
// residual stream
// ---------------------------------------------------------------------------
enum { kGateNone = 0, kGateVector = 1, kGateSequence = 2, kGateToken = 3 };
struct ResidualArgs {
    int B, T, d, post, pre, gate;  // gate: kGate*
    bool has_y, has_dh;
    float ra, rb, eps;  // residual and branch scale
    Rows x, y, g, h, n;      // forward: h, n written; backward: their gradients
    Rows dx, dy, dg;
    const void *wpost, *wpre;
};
size_t residual_scratch_bytes(int dtype, const ResidualArgs& a);
int launch_residual_norm(int dtype, const ResidualArgs& a, hipStream_t stream);
int launch_residual_norm_bwd(int dtype, const ResidualArgs& a, void* dwpost, bool dgate, void* dwpre, void* scratch,
                             hipStream_t stream);

// ---------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------
enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };
struct Matrix {
    char* p;
    int64_t row;  // elements from one row to the next
};
struct LinearArgs {
    int M, K, N, act, out_in;  // rows, d_in, d_out
    Matrix x, w, r, y, z, dy, dx, dw;
    const void* b;
    void* db;
};
size_t linear_fwd_scratch(int dtype, const LinearArgs& a);
size_t linear_bwd_scratch(int dtype, const LinearArgs& a);
int launch_linear(int dtype, const LinearArgs& a, void* scratch, hipStream_t stream);
int launch_linear_bwd(int dtype, const LinearArgs& a, void* scratch, hipStream_t stream);

// ---------------------------------------------------------------------------
// log probabilities
// ---------------------------------------------------------------------------
constexpr int kMaxTop = 32;
struct LogprobArgs {
    int R, V, top;
    float scale;
    const char* x;
    int64_t row;
    const int32_t* target;
    float *logp, *lse, *stats, *entropy, *top_logp;
    int32_t* top_index;
    const float *dlogp, *dlse, *dent;
    char* dx;
    int64_t drow;
};
size_t logprob_scratch_bytes(int dtype, int R, int V, int top);
int launch_logprobs(int dtype, const LogprobArgs& a, void* scratch, hipStream_t stream);
int launch_logprobs_bwd(int dtype, const LogprobArgs& a, hipStream_t stream);

}  // namespace mosa
