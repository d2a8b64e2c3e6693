// Argument checks that the operators' C entries share.
#pragma once

#include "heads.h"
#include "mosa.h"

namespace mosa {

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline int elem_size(int dtype) { return dtype == MOSA_BF16 ? 2 : 4; }
inline bool dtype_ok(int dtype) { return dtype == MOSA_BF16 || dtype == MOSA_F32; }

// Rows counted in 32 bits by the kernels (offsets into tensors are 64-bit).
inline bool rows_ok(int64_t a, int64_t b, int64_t c) { return (double)a * (double)b * (double)c <= 2147483647.0; }

// Nothing on a device reaches over more; within it offsets and sizes in bytes stay far
// from 64 bits.
constexpr double kMostBytes = 70368744177664.0;  // 2^46

// One tensor of rows [B, H, T, dh]: address and strides checked and taken over.
inline int take_rows(const mosa_rows* r, int B, int H, int T, int dh, int dtype, bool output, Rows* to) {
    if (!r || !r->data || !aligned(r->data, 16)) return MOSA_ERR_INVALID_ARG;
    const int64_t unit = 16 / elem_size(dtype);
    const int n[3] = {B, H, T};
    int64_t st[3] = {r->batch_stride, r->head_stride, r->row_stride};
    double span = 0.0;  // from the first row to the last
    for (int i = 0; i < 3; ++i) {
        if (n[i] == 1) st[i] = 0;
        // (a stride beyond 2^40 elements is no tensor of this device)
        if (st[i] < 0 || st[i] % unit || st[i] > ((int64_t)1 << 40)) return MOSA_ERR_INVALID_ARG;
        span += (double)(n[i] - 1) * (double)st[i];
    }
    if (span * elem_size(dtype) > kMostBytes) return MOSA_ERR_INVALID_ARG;
    if (output) {  // nested axes: each stride at least the extent of those within
        int64_t extent = dh;
        bool used[3] = {false, false, false};
        for (int i = 0; i < 3; ++i) {
            int m = -1;
            for (int j = 0; j < 3; ++j)
                if (!used[j] && (m < 0 || st[j] < st[m])) m = j;
            used[m] = true;
            if (n[m] == 1) continue;
            if (st[m] < extent) return MOSA_ERR_INVALID_ARG;
            extent += (n[m] - 1) * st[m];
        }
    }
    *to = Rows{static_cast<char*>(r->data), st[0], st[1], st[2]};
    return MOSA_OK;
}

inline int check_scratch(const void* scratch, size_t have, size_t need) {
    if (need == 0) return MOSA_OK;
    if (!scratch || !aligned(scratch, 256)) return MOSA_ERR_INVALID_ARG;
    return have < need ? MOSA_ERR_WORKSPACE : MOSA_OK;
}

inline int done(int e) { return e ? MOSA_ERR_HIP : MOSA_OK; }

}  // namespace mosa
