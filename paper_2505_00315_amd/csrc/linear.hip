// Product with a weight matrix, its epilogue, and its gradients.
//
//   y = act(x w + b) + r;   dz = dy act'(z),  dx = dz w^T,  dw = x^T dz,  db = sum dz
//
// Three products of 2 rows d_in d_out operations each (prod.h); dz and db are one
// pass over dy and z before them.
#include "prod.h"

namespace mosa {

namespace {

// dz = dy act'(z) (where there is an activation) and partial sums of it over rows:
// 32 units of columns by 8 rows of lanes, a run of rows per workgroup.
template <typename ST>
__global__ __launch_bounds__(256) void linear_dz_kernel(LinearArgs a, int per, ST* __restrict__ dz, WideSum<ST>* __restrict__ part) {
    constexpr int E = Unit<ST>::E;
    __shared__ WideSum<ST> red[8][32 * E + 1];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, n = (blockIdx.x * 32 + tx) * E;
    const int64_t r0 = (int64_t)blockIdx.y * per, r1 = r0 + per < a.M ? r0 + per : a.M;
    WideSum<ST> s[E];
#pragma unroll
    for (int e = 0; e < E; ++e) s[e] = 0;
    if (n < a.N) {
#pragma unroll 4
        for (int64_t r = r0 + ty; r < r1; r += 8) {
            Unit<ST> u;
            float d[E];
            u.load(reinterpret_cast<const ST*>(a.dy.p) + r * a.dy.row + n);
            u.get(d);
            if (a.act) {
                float z[E];
                u.load(reinterpret_cast<const ST*>(a.z.p) + r * a.z.row + n);
                u.get(z);
#pragma unroll
                for (int e = 0; e < E; ++e) d[e] *= act_slope<ST>(z[e], a.act);
                u.set(d);
                u.store(dz + r * a.N + n);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) s[e] += d[e];
        }
    }
    if (!part) return;
#pragma unroll
    for (int e = 0; e < E; ++e) red[ty][tx * E + e] = s[e];
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * E; i += 256) {
        const int col = blockIdx.x * 32 * E + i;
        WideSum<ST> t = 0;
        for (int k = 0; k < 8; ++k) t += red[k][i];
        if (col < a.N) part[(size_t)blockIdx.y * a.N + col] = t;
    }
}

struct DzSplit {
    int gx, parts, per;
};
DzSplit dz_split(int dtype, const LinearArgs& a) {
    const int wide = 32 * 16 / (dtype == kBF16 ? 2 : 4);  // columns of a workgroup
    DzSplit s;
    s.gx = (a.N + wide - 1) / wide;
    const int64_t want = (2048 + s.gx - 1) / s.gx, most = (a.M + 31) / 32;
    const int64_t parts = want < most ? want : most;
    s.per = (int)((a.M + parts - 1) / parts);
    s.parts = (a.M + s.per - 1) / s.per;
    return s;
}

// Tiles of a product and what they take: us per chunk of k for a workgroup that has a CU to itself and for one of a
// full CU, us at its ends, workgroups that fit a CU.  Measured (bf16, TFLOP/s): 256 x 256 tiles 1330 for 16384 x 8192
// by 4096; 128 x 128 1080 there and 1120 for 8192 x 4096 by 1024, where the large ones leave half the CUs idle (820);
// its form with more stages for one workgroup per CU 980 against 830 (1024 x 8192 by 4096); 64 x 64 670 against 410
// and 540 of the others (2048 x 4096 by 1024).  fp32: 64 x 64 148 for 4096^3, and 32 x 32 130 there and 64 against 47
// for 777 x 520 by 1304.
struct TileKind {
    int size;
    float alone, full, ends;
    int fit;
};
constexpr TileKind kTilesBf16[] = {{256, 1.61f, 1.61f, 7.f, 1}, {128, 0.66f, 0.495f, 1.7f, 2}, {128, 0.54f, 0.54f, 2.f, 1},
                                   {64, 0.28f, 0.20f, 2.5f, 2}};
constexpr TileKind kTilesF32[] = {{64, 0.65f, 0.50f, 2.5f, 4}, {32, 0.36f, 0.17f, 2.5f, 4}};
constexpr int kCus = 256;

// How a product is computed: kind of tiles, parts of K and k of each; rows: few rows, one launch.
struct Plan {
    int kind, size, splits, kper;
    bool rows;
};
Plan plan_of(int dtype, int M, int N, int K, bool kcontig) {
    const int kc = dtype == kBF16 ? 64 : 32, es = dtype == kBF16 ? 2 : 4;
    const int64_t chunks = (K + kc - 1) / kc;
    // Few rows by a k-contiguous weight: one launch where its workgroups are enough to read the weight at the memory's rate.
    if (kcontig && M <= 32 && N >= 96 * 16) return {0, 0, 1, K, true};
    const TileKind* kinds = dtype == kBF16 ? kTilesBf16 : kTilesF32;
    const int count = dtype == kBF16 ? 4 : 2;
    Plan best{};
    float least = 0.f;
    for (int k = 0; k < count; ++k) {
        const TileKind& t = kinds[k];
        const int64_t tiles = (int64_t)((M + t.size - 1) / t.size) * ((N + t.size - 1) / t.size);
        for (int splits = 1; splits <= 16; ++splits) {
            const int64_t per = (chunks + splits - 1) / splits;
            if (splits > 1 && (per < 4 || (chunks + per - 1) / per != splits)) continue;
            const int64_t n = (tiles * splits + kCus - 1) / kCus;  // workgroups of a CU
            const float chunk = t.alone > n * t.full ? t.alone : n * t.full;
            float time = chunk * per + t.ends * ((n + t.fit - 1) / t.fit);
            // the parts' sum: another launch, and its bytes at the rate of the last cache
            if (splits > 1) time += 6.f + (float)splits * M * N * 8.f / 7e6f;
            if (least == 0.f || time < least) least = time, best = {k, t.size, splits, (int)per * kc, false};
        }
    }
    return best;
}
size_t part_bytes(const Plan& p, int M, int N) { return p.splits > 1 ? (size_t)p.splits * M * N * sizeof(float) : 0; }

template <typename ST, bool PKC, bool QKC>
int product(ProdArgs a, const Plan& p, hipStream_t stream) {
    if constexpr (PKC && QKC) {
        if (p.rows) {
            // Two workgroups of 4 waves per CU where there are enough of them: one's start and end beside the other's loads.
            if (a.N >= 2 * kCus * 16)
                return a.M <= 16 ? launch_prod_rows<ST, 1, 4>(a, stream) : launch_prod_rows<ST, 2, 4>(a, stream);
            return a.M <= 16 ? launch_prod_rows<ST, 1, 8>(a, stream) : launch_prod_rows<ST, 2, 8>(a, stream);
        }
    }
    a.tn = (a.N + p.size - 1) / p.size, a.tm = (a.M + p.size - 1) / p.size;
    a.splits = p.splits, a.kper = p.kper;
    if constexpr (sizeof(ST) == 2) {
        switch (p.kind) {
            case 0: return launch_prod<ProdShape<ST, PKC, QKC, 256, 256, 2, 4, 2, 2>>(a, stream);
            case 1: return launch_prod<ProdShape<ST, PKC, QKC, 128, 128, 2, 2, 2>>(a, stream);
            case 2: return launch_prod<ProdShape<ST, PKC, QKC, 128, 128, 2, 4, 4>>(a, stream);
            default: return launch_prod<ProdShape<ST, PKC, QKC, 64, 64, 2, 2, 4>>(a, stream);
        }
    } else {
        if (p.kind == 0) return launch_prod<ProdShape<ST, PKC, QKC, 64, 64, 2, 2, 2>>(a, stream);
        return launch_prod<ProdShape<ST, PKC, QKC, 32, 32, 2, 2, 2>>(a, stream);
    }
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

template <typename ST>
int forward_t(int dtype, const LinearArgs& a, void* scratch, hipStream_t stream) {
    ProdArgs p{};
    p.p = a.w.p, p.q = a.x.p, p.prow = a.w.row * (int64_t)sizeof(ST), p.qrow = a.x.row * (int64_t)sizeof(ST);
    p.M = a.M, p.N = a.N, p.K = a.K;
    p.part = static_cast<float*>(scratch);
    p.bias = a.b, p.act = a.act, p.r = a.r, p.y = a.y, p.z = a.z;
    const Plan plan = plan_of(dtype, a.M, a.N, a.K, a.out_in);
    return a.out_in ? product<ST, true, true>(p, plan, stream) : product<ST, false, true>(p, plan, stream);
}

struct BwdScratch {  // offsets in bytes
    size_t dz, sums, part, total;
};
BwdScratch bwd_scratch(int dtype, const LinearArgs& a) {
    BwdScratch s{};
    const size_t es = dtype == kBF16 ? 2 : 4;
    s.sums = a.act ? round256((size_t)a.M * a.N * es) : 0;
    s.part = s.sums + round256((size_t)dz_split(dtype, a).parts * a.N * wide_sum_bytes(dtype));
    const size_t dx = part_bytes(plan_of(dtype, a.M, a.K, a.N, !a.out_in), a.M, a.K);
    const size_t dw = part_bytes(a.out_in ? plan_of(dtype, a.N, a.K, a.M, false) : plan_of(dtype, a.K, a.N, a.M, false), a.K, a.N);
    s.total = s.part + (dx > dw ? dx : dw);
    return s;
}

template <typename ST>
int backward_t(int dtype, const LinearArgs& a, void* scratch, hipStream_t stream) {
    char* at = static_cast<char*>(scratch);
    const BwdScratch s = bwd_scratch(dtype, a);
    float* part = reinterpret_cast<float*>(at + s.part);
    Matrix dz = a.dy;
    if (a.act || a.db) {
        const DzSplit d = dz_split(dtype, a);
        WideSum<ST>* sums = a.db ? reinterpret_cast<WideSum<ST>*>(at + s.sums) : nullptr;
        ST* out = reinterpret_cast<ST*>(at + s.dz);
        hipLaunchKernelGGL((linear_dz_kernel<ST>), dim3(d.gx, d.parts), dim3(256), 0, stream, a, d.per, out, sums);
        if (hipGetLastError() != hipSuccess) return -1;
        if (a.db && launch_sum_parts(dtype, SumParts{sums, d.parts, 1, a.N, {a.db, nullptr, nullptr}}, stream)) return -1;
        if (a.act) dz = Matrix{at + s.dz, a.N};
    }
    const int64_t es = sizeof(ST);
    if (a.dx.p) {  // dz [M, N] by w^T: k is w's d_out axis
        ProdArgs p{};
        p.p = a.w.p, p.prow = a.w.row * es, p.q = dz.p, p.qrow = dz.row * es;
        p.M = a.M, p.N = a.K, p.K = a.N, p.part = part, p.y = a.dx;
        const Plan plan = plan_of(dtype, p.M, p.N, p.K, !a.out_in);
        if (a.out_in ? product<ST, false, true>(p, plan, stream) : product<ST, true, true>(p, plan, stream)) return -1;
    }
    if (a.dw.p) {  // x^T dz, or dz^T x where w's rows are outputs
        const Matrix &rows = a.out_in ? dz : a.x, &cols = a.out_in ? a.x : dz;
        ProdArgs p{};
        p.p = cols.p, p.prow = cols.row * es, p.q = rows.p, p.qrow = rows.row * es;
        p.M = a.out_in ? a.N : a.K, p.N = a.out_in ? a.K : a.N, p.K = a.M, p.part = part, p.y = a.dw;
        if (product<ST, false, false>(p, plan_of(dtype, p.M, p.N, p.K, false), stream)) return -1;
    }
    return 0;
}

}  // namespace

size_t linear_fwd_scratch(int dtype, const LinearArgs& a) { return part_bytes(plan_of(dtype, a.M, a.N, a.K, a.out_in), a.M, a.N); }
size_t linear_bwd_scratch(int dtype, const LinearArgs& a) { return bwd_scratch(dtype, a).total; }

int launch_linear(int dtype, const LinearArgs& a, void* scratch, hipStream_t stream) {
    return dtype == kBF16 ? forward_t<uint16_t>(dtype, a, scratch, stream) : forward_t<float>(dtype, a, scratch, stream);
}

int launch_linear_bwd(int dtype, const LinearArgs& a, void* scratch, hipStream_t stream) {
    return dtype == kBF16 ? backward_t<uint16_t>(dtype, a, scratch, stream) : backward_t<float>(dtype, a, scratch, stream);
}

}  // namespace mosa
