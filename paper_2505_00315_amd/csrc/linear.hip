// Product with a weight matrix, its epilogue, and its gradients.
//
//   y = act(x w + b) + r;   dz = dy act'(z),  dx = dz w^T,  dw = x^T dz,  db = sum dz
//
// Three products of 2 rows d_in d_out operations each (prod.h); dz and db are one
// pass over dy and z before them (8192 x 4096 bf16: 48 us for 204 MB, 4.2 TB/s, with
// gelu's slope; dy alone 28 us for 136 MB).
//
// Measured (bf16, 16384 rows, 8192 by 4096): forward 885 us, dx 899, dw 839, 1220 to
// 1310 TFLOP/s (a library product of the same sizes 1341, of 8192^3 1387).
#include "prod.h"

namespace mosa {

namespace {

// dz = dy act'(z) (where there is an activation) and partial sums of it over rows:
// 32 units of columns by 8 rows of lanes, a run of rows per workgroup.  dz is kept in
// storage type: with bf16 it is rounded once, as the matrix instruction takes bf16
// operands only and two of them, dz and what its rounding leaves, would double both
// products (some 125 us more for 8192 x 1024 by 4096).  So dx and dw are 0.0024 off
// 64-bit results, 0.0017 without that rounding and z's, and 1.4e-4 off a form that
// makes the two; db is the sum of dz before it is rounded.
template <typename ST>
__global__ __launch_bounds__(256) void linear_dz_kernel(LinearArgs a, int per, ST* __restrict__ dz, WideSum<ST>* __restrict__ part) {
    constexpr int E = Unit<ST>::E, U = 4;
    __shared__ WideSum<ST> red[8][32 * E + 1];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, n = (blockIdx.x * 32 + tx) * E;
    const int64_t r0 = (int64_t)blockIdx.y * per, r1 = r0 + per < a.M ? r0 + per : a.M;
    WideSum<ST> s[E];
#pragma unroll
    for (int e = 0; e < E; ++e) s[e] = 0;
    if (n < a.N) {
        for (int64_t r = r0 + ty; r < r1; r += 8 * U) {
            Unit<ST> y[U], z[U];  // U rows' loads together (a past row's: the last one's again)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t at = r + 8 * u < r1 ? r + 8 * u : r1 - 1;
                y[u].load(reinterpret_cast<const ST*>(a.dy.p) + at * a.dy.row + n);
                if (a.act) z[u].load(reinterpret_cast<const ST*>(a.z.p) + at * a.z.row + n);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (r + 8 * u >= r1) break;
                float d[E];
                y[u].get(d);
                if (a.act) {
                    float v[E];
                    z[u].get(v);
                    times_slope<ST>(d, v, a.act);
                    Unit<ST> o;
                    o.set(d);
                    o.store(dz + (r + 8 * u) * a.N + n);
                }
#pragma unroll
                for (int e = 0; e < E; ++e) s[e] += d[e];
            }
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
constexpr TileKind kTilesBf16[] = {{256, 1.55f, 1.55f, 6.f, 1}, {128, 0.66f, 0.495f, 1.7f, 2}, {128, 0.49f, 0.49f, 4.5f, 1},
                                   {64, 0.28f, 0.20f, 2.5f, 2}};
constexpr TileKind kTilesF32[] = {{64, 0.65f, 0.50f, 2.5f, 4}, {32, 0.36f, 0.17f, 2.5f, 4}};

int kinds_of(int dtype) { return dtype == kBF16 ? 4 : 2; }
const TileKind& kind_of(int dtype, int k) { return dtype == kBF16 ? kTilesBf16[k] : kTilesF32[k]; }
int64_t tiles_of(int M, int N, int size) { return (int64_t)((M + size - 1) / size) * ((N + size - 1) / size); }

// How a product is computed: kind of tiles, parts of K and k of each; rows: few rows, one launch.
struct Plan {
    int kind, size, splits, kper;
    bool rows;
};
// This kind and number of parts (splits 0: not one that there is).
Plan tiled(int dtype, int M, int N, int K, int kind, int splits) {
    const int kc = dtype == kBF16 ? 64 : 32, chunks = (K + kc - 1) / kc, per = (chunks + splits - 1) / splits;
    if (splits > 1 && (per < 4 || (chunks + per - 1) / per != splits)) return {};
    return {kind, kind_of(dtype, kind).size, splits, per * kc, false};
}
// The parts' sum: another launch, and its bytes at the rate of the last cache.
float join_time(const Plan& p, int M, int N) { return p.splits > 1 ? 5.f + (float)p.splits * M * N * 8.f / 5e6f : 0.f; }
// A chunk of each of the n workgroups of a CU: two at a time, or all beside each other.
float chunk_time(const TileKind& t, int64_t n) {
    if (t.fit == 2) return (float)(n / 2) * 2.f * t.full + (float)(n % 2) * t.alone;
    return t.alone > n * t.full ? t.alone : n * t.full;
}

// Few rows by strips of a weight with its columns along its rows: us for the k of a strip, one strip of a CU after the
// other.  Measured with 1, 16 and 32 rows (us; tiles): bf16 512 x 2048 3.4, 3.5, 3.8 (4.5, 4.6, 4.8), 1024 x 4096 6.4, 6.7,
// 7.2 (7.3, 7.6, 8.1), 4096 x 4096 17, 18, 20 (14, 15, 13); fp32 512 x 2048 4.4, 4.7, 6.0 (9.0, 9.2, 9.3), 1024 x 4096 7.8, 8.1,
// 10.6 (9.8, 10.9, 11.4), 4096 x 8192 30, 29, 33 (47, 47, 48), 4096 x
// 16384 56, 58, 64 (86).
constexpr int kStrip = 32;  // columns
float strips_time(int dtype, int M, int N, int K) {
    const float per_k = dtype == kBF16 ? (M <= 16 ? 0.0041f : 0.0047f) : M <= 16 ? 0.0050f : 0.0062f;
    const int64_t strips = ((int64_t)N + kStrip - 1) / kStrip;
    return 2.f + (float)((strips + kCus - 1) / kCus) * K * per_k;
}

// What lies k-contiguous of a product's sides: both (the weight is the n side), the m side, or neither.
enum class Layout { kBoth, kRows, kNone };

// time: what the plan is taken to need, us.
Plan plan_of(int dtype, int M, int N, int K, Layout layout, float* time = nullptr) {
    const int kc = dtype == kBF16 ? 64 : 32;
    // Few rows by a k-contiguous weight: one launch where its workgroups are enough to read the weight at the memory's rate.
    if (layout == Layout::kBoth && M <= 32 && N >= 96 * 16) {
        if (time) *time = 0.f;  // (never paired)
        return {0, 0, 1, K, true};
    }
    // No kind is faster than memory (a few rows by a weight of 16384 x 4096: 31 us with one workgroup for every CU, 38 with
    // the two that would be enough for twice the products).
    const float bytes = (float)(dtype == kBF16 ? 2 : 4) * ((float)M * K + (float)K * N + (float)M * N), floor = bytes / 5.2e6f;
    Plan best{};
    float least = 0.f;
    for (int k = 0; k < kinds_of(dtype); ++k) {
        const TileKind& t = kind_of(dtype, k);
        const int64_t tiles = tiles_of(M, N, t.size);
        for (const int splits : {1, 2, 3, 4, 6, 8, 12, 16}) {
            const Plan p = tiled(dtype, M, N, K, k, splits);
            if (!p.splits) continue;
            const int64_t n = (tiles * splits + kCus - 1) / kCus;  // workgroups of a CU
            const float alone = chunk_time(t, n) * (p.kper / kc) + t.ends * ((n + t.fit - 1) / t.fit);
            const float taken = (alone > floor ? alone : floor) + join_time(p, M, N);
            if (least == 0.f || taken < least) least = taken, best = p;
        }
    }
    if (layout == Layout::kRows && M <= 32) {
        // fp32 tiles have a quarter of the bytes of others in flight: weights of 4096 x 8192 to 16384 x 4096 at 2.9 to 3.1 TB/s.
        if (dtype != kBF16 && least < bytes / 3.1e6f) least = bytes / 3.1e6f;
        const float strips = strips_time(dtype, M, N, K), taken = strips > floor ? strips : floor;
        if (taken < least) least = taken, best = {0, 0, 1, K, true};
    }
    if (time) *time = least;
    return best;
}
// x w and dz w^T
Layout forward_layout(const LinearArgs& a) { return a.out_in ? Layout::kBoth : Layout::kRows; }
Layout dx_layout(const LinearArgs& a) { return a.out_in ? Layout::kRows : Layout::kBoth; }
size_t part_bytes(const Plan& p, int M, int N) { return p.splits > 1 ? (size_t)p.splits * M * N * sizeof(float) : 0; }

// The tile shape of a kind.
template <typename ST, bool PKC, bool QKC, int KIND>
auto shape_of() {
    if constexpr (sizeof(ST) == 2) {
        if constexpr (KIND == 0) return ProdShape<ST, PKC, QKC, 256, 256, 2, 4, 2, 2>{};
        else if constexpr (KIND == 1) return ProdShape<ST, PKC, QKC, 128, 128, 2, 2, 2>{};
        else if constexpr (KIND == 2) return ProdShape<ST, PKC, QKC, 128, 128, 2, 4, 4>{};
        else return ProdShape<ST, PKC, QKC, 64, 64, 2, 2, 4>{};
    } else {
        if constexpr (KIND == 0) return ProdShape<ST, PKC, QKC, 64, 64, 2, 2, 2>{};
        else return ProdShape<ST, PKC, QKC, 32, 32, 2, 2, 2>{};
    }
}
template <typename ST, bool PKC, bool QKC, int KIND>
using ShapeOf = decltype(shape_of<ST, PKC, QKC, KIND>());

void take_plan(ProdArgs& a, const Plan& p) {
    a.tn = (a.N + p.size - 1) / p.size, a.tm = (a.M + p.size - 1) / p.size;
    a.splits = p.splits, a.kper = p.kper;
}

template <typename ST, bool PKC, bool QKC>
int product(ProdArgs a, const Plan& p, hipStream_t stream) {
    if constexpr (PKC && QKC) {
        if (p.rows) {
            // Two workgroups of 4 waves per CU where there are enough of them: one's start and end beside the other's loads.
            if (a.N >= 2 * kCus * 16)
                return a.M <= 16 ? launch_prod_rows<ProdRows<ST, true, 16, 1, 4>, 4>(a, stream)
                                 : launch_prod_rows<ProdRows<ST, true, 16, 2, 3>, 4>(a, stream);
            return a.M <= 16 ? launch_prod_rows<ProdRows<ST, true, 16, 1, 4>, 8>(a, stream)
                             : launch_prod_rows<ProdRows<ST, true, 16, 2, 3>, 8>(a, stream);
        }
    }
    if constexpr (!PKC && QKC) {
        if (p.rows)
            return a.M <= 16 ? launch_prod_rows<ProdRows<ST, false, kStrip, 1, 2>, 8>(a, stream)
                             : launch_prod_rows<ProdRows<ST, false, kStrip, 2, 2>, 8>(a, stream);
    }
    take_plan(a, p);
    if constexpr (sizeof(ST) == 2) {
        if (p.kind == 0) return launch_prod<ShapeOf<ST, PKC, QKC, 0>>(a, stream);
        if (p.kind == 1) return launch_prod<ShapeOf<ST, PKC, QKC, 1>>(a, stream);
        if (p.kind == 2) return launch_prod<ShapeOf<ST, PKC, QKC, 2>>(a, stream);
        return launch_prod<ShapeOf<ST, PKC, QKC, 3>>(a, stream);
    } else {
        if (p.kind == 0) return launch_prod<ShapeOf<ST, PKC, QKC, 0>>(a, stream);
        return launch_prod<ShapeOf<ST, PKC, QKC, 1>>(a, stream);
    }
}

// dx and dw of a call, and the plans of both: one launch for the two (and for db's sum) where that is taken to be
// shorter than one after the other (a launch that waits for another starts some 4 us late, and each leaves CUs idle
// at its end).
struct BwdPlan {
    Plan dx, dw;    // alone
    bool pair;
    Plan dx2, dw2;  // in one launch
};
// The products' sizes: dx [M, K] over N; dw [K, N] or [N, K] over M.
struct Size {
    int M, N, K;
};
Size dx_size(const LinearArgs& a) { return {a.M, a.K, a.N}; }
Size dw_size(const LinearArgs& a) { return a.out_in ? Size{a.N, a.K, a.M} : Size{a.K, a.N, a.M}; }
BwdPlan plan_bwd(int dtype, const LinearArgs& a) {
    const Size x = dx_size(a), w = dw_size(a);
    float tx, tw;
    BwdPlan best{plan_of(dtype, x.M, x.N, x.K, dx_layout(a), &tx), plan_of(dtype, w.M, w.N, w.K, Layout::kNone, &tw), false, {}, {}};
    if (best.dx.rows) return best;
    float least = tx + tw + 6.f;
    const int kc = dtype == kBF16 ? 64 : 32;
    for (int k = 0; k < kinds_of(dtype); ++k) {
        const TileKind& t = kind_of(dtype, k);
        if (dtype == kBF16 && k % 2 == 0) continue;  // (workgroups of 4 waves; the large tiles' products are long)
        const int64_t tx1 = tiles_of(x.M, x.N, t.size), tw1 = tiles_of(w.M, w.N, t.size);
        for (const int sx : {1, 2, 4}) {
            const Plan p = tiled(dtype, x.M, x.N, x.K, k, sx);
            if (!p.splits) continue;
            for (const int sw : {1, 2, 3, 4, 6, 8, 12, 16}) {
                const Plan q = tiled(dtype, w.M, w.N, w.K, k, sw);
                if (!q.splits) continue;
                const int64_t bx = tx1 * sx, bw = tw1 * sw;
                const float cx = (float)p.kper / kc, cw = (float)q.kper / kc, longest = cx > cw ? cx : cw;
                const int64_t n = (bx + bw + kCus - 1) / kCus;
                // a CU's share, in whole workgroups, and the longest workgroup
                const float share = t.full * (bx * cx + bw * cw) / (float)(bx + bw) * n, alone = t.alone * longest;
                const float jx = join_time(p, x.M, x.N), jw = join_time(q, w.M, w.N);
                const float join = jx > 0.f && jw > 0.f ? jx + jw - 5.f : jx + jw;
                const float time = (share > alone ? share : alone) + t.ends * ((n + t.fit - 1) / t.fit) + join;
                if (time < least) least = time, best.pair = true, best.dx2 = p, best.dw2 = q;
            }
        }
    }
    return best;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

template <typename ST>
int forward_t(int dtype, const LinearArgs& a, void* scratch, hipStream_t stream) {
    ProdArgs p{};
    p.p = a.w.p, p.q = a.x.p, p.prow = a.w.row * (int64_t)sizeof(ST), p.qrow = a.x.row * (int64_t)sizeof(ST);
    p.M = a.M, p.N = a.N, p.K = a.K;
    p.part = static_cast<float*>(scratch);
    p.bias = a.b, p.act = a.act, p.r = a.r, p.y = a.y, p.z = a.z;
    const Plan plan = plan_of(dtype, a.M, a.N, a.K, forward_layout(a));
    return a.out_in ? product<ST, true, true>(p, plan, stream) : product<ST, false, true>(p, plan, stream);
}

struct BwdScratch {  // offsets in bytes
    size_t dz, sums, part, total;
    BwdPlan plan;
};
BwdScratch bwd_scratch(int dtype, const LinearArgs& a) {
    BwdScratch s{};
    const size_t es = dtype == kBF16 ? 2 : 4;
    s.sums = a.act ? round256((size_t)a.M * a.N * es) : 0;
    s.part = s.sums + round256((size_t)dz_split(dtype, a).parts * a.N * wide_sum_bytes(dtype));
    const Size x = dx_size(a), w = dw_size(a);
    s.plan = plan_bwd(dtype, a);
    // one product after the other, as also where a call wants one only; or both at once
    const size_t dx = part_bytes(s.plan.dx, x.M, x.N), dw = part_bytes(s.plan.dw, w.M, w.N), one = dx > dw ? dx : dw;
    const size_t both = s.plan.pair ? round256(part_bytes(s.plan.dx2, x.M, x.N)) + part_bytes(s.plan.dw2, w.M, w.N) : 0;
    s.total = s.part + (both > one ? both : one);
    return s;
}

template <typename ST, bool OUT_IN, int KIND>
int product_pair(const ProdPair& p, hipStream_t stream) {
    return launch_prod_pair<ShapeOf<ST, !OUT_IN, true, KIND>, ShapeOf<ST, false, false, KIND>>(p, stream);
}

template <typename ST>
int backward_t(int dtype, const LinearArgs& a, void* scratch, hipStream_t stream) {
    char* at = static_cast<char*>(scratch);
    const BwdScratch s = bwd_scratch(dtype, a);
    float* part = reinterpret_cast<float*>(at + s.part);
    Matrix dz = a.dy;
    SumParts db{};
    if (a.act || a.db) {
        const DzSplit d = dz_split(dtype, a);
        WideSum<ST>* sums = a.db ? reinterpret_cast<WideSum<ST>*>(at + s.sums) : nullptr;
        ST* out = reinterpret_cast<ST*>(at + s.dz);
        hipLaunchKernelGGL((linear_dz_kernel<ST>), dim3(d.gx, d.parts), dim3(256), 0, stream, a, d.per, out, sums);
        if (hipGetLastError() != hipSuccess) return -1;
        if (a.act) dz = Matrix{at + s.dz, a.N};
        db = SumParts{sums, d.parts, a.db ? 1 : 0, a.N, {a.db, nullptr, nullptr}};
    }
    const int64_t es = sizeof(ST);
    ProdArgs x{}, w{};
    const Size sx = dx_size(a), sw = dw_size(a);
    // dz by w^T: k is w's d_out axis
    x.p = a.w.p, x.prow = a.w.row * es, x.q = dz.p, x.qrow = dz.row * es;
    x.M = sx.M, x.N = sx.N, x.K = sx.K, x.part = part, x.y = a.dx;
    // x^T dz, or dz^T x where w's rows are outputs
    const Matrix &rows = a.out_in ? dz : a.x, &cols = a.out_in ? a.x : dz;
    w.p = cols.p, w.prow = cols.row * es, w.q = rows.p, w.qrow = rows.row * es;
    w.M = sw.M, w.N = sw.N, w.K = sw.K, w.part = part, w.y = a.dw;
    if (a.dx.p && a.dw.p && s.plan.pair) {
        const Plan &px = s.plan.dx2, &pw = s.plan.dw2;
        take_plan(x, px), take_plan(w, pw);
        w.part = reinterpret_cast<float*>(at + s.part + round256(part_bytes(px, x.M, x.N)));
        const ProdPair p{x, w, db, 0, 0, false};
        constexpr int FIRST = sizeof(ST) == 2 ? 1 : 0, SECOND = sizeof(ST) == 2 ? 3 : 1;
        if (px.kind == FIRST) return a.out_in ? product_pair<ST, true, FIRST>(p, stream) : product_pair<ST, false, FIRST>(p, stream);
        return a.out_in ? product_pair<ST, true, SECOND>(p, stream) : product_pair<ST, false, SECOND>(p, stream);
    }
    if (db.n && launch_sum_parts(dtype, db, stream)) return -1;
    if (a.dx.p)
        if (a.out_in ? product<ST, false, true>(x, s.plan.dx, stream) : product<ST, true, true>(x, s.plan.dx, stream)) return -1;
    return a.dw.p ? product<ST, false, false>(w, s.plan.dw, stream) : 0;
}

}  // namespace

size_t linear_fwd_scratch(int dtype, const LinearArgs& a) { return part_bytes(plan_of(dtype, a.M, a.N, a.K, forward_layout(a)), a.M, a.N); }
size_t linear_bwd_scratch(int dtype, const LinearArgs& a) { return bwd_scratch(dtype, a).total; }

int launch_linear(int dtype, const LinearArgs& a, void* scratch, hipStream_t stream) {
    return dtype == kBF16 ? forward_t<uint16_t>(dtype, a, scratch, stream) : forward_t<float>(dtype, a, scratch, stream);
}

int launch_linear_bwd(int dtype, const LinearArgs& a, void* scratch, hipStream_t stream) {
    return dtype == kBF16 ? backward_t<uint16_t>(dtype, a, scratch, stream) : backward_t<float>(dtype, a, scratch, stream);
}

}  // namespace mosa
