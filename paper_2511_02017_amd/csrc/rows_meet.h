// Whether two tensors of rows share memory: host code.
#pragma once

#include <algorithm>
#include <cstdint>

#include "tapout.h"

namespace tapout {

// x and y: B x K rows of V elements, strides from 0 on; those of y lie apart, all of a run of one axis before the next run, those of x anyhow.  Tensors that lie
// beside each other are told apart by their ends, rows between each other's rows one by one.
inline bool rows_meet(const tapout_logits &x, const tapout_logits &y, int B, int K, int V)
{
    const auto bytes = [](const tapout_logits &t) { return t.dtype == TAPOUT_F32 ? 4 : 2; };
    // strides in bytes; of an axis of one row: none
    const int64_t xb = B > 1 ? x.stride_b * bytes(x) : 0, xk = K > 1 ? x.stride_k * bytes(x) : 0, len_x = (int64_t)V * bytes(x);
    const int64_t yb = B > 1 ? y.stride_b * bytes(y) : 0, yk = K > 1 ? y.stride_k * bytes(y) : 0, len_y = (int64_t)V * bytes(y);
    const int64_t x0 = (int64_t)((uintptr_t)x.ptr - (uintptr_t)y.ptr);                     // from y's first row on
    if (x0 >= (B - 1) * yb + (K - 1) * yk + len_y || x0 + (B - 1) * xb + (K - 1) * xk + len_x <= 0) return false;
    // rows of y by their address: runs of the axis with the smaller stride
    const bool k_inner = yk <= yb || B == 1;
    const int64_t outer = std::max<int64_t>(k_inner ? yb : yk, 1), inner = std::max<int64_t>(k_inner ? yk : yb, 1);
    const int64_t outers = k_inner ? B : K, inners = k_inner ? K : B;
    for (int b = 0; b < B; ++b)
        for (int k = 0; k < K; ++k) {
            const int64_t begin = x0 + b * xb + k * xk, last = begin + len_x - 1;
            if (last < 0) continue;
            // the last row of y that begins up to this row's last byte; if that ends before this row, so do all before it
            const int64_t o = std::min(last / outer, outers - 1), i = std::min((last - o * outer) / inner, inners - 1);
            if (o * outer + i * inner + len_y > begin) return true;
        }
    return false;
}

}  // namespace tapout
