// cf_native.h -- what the sources of the module _cf_args share.
#pragma once

#include <ATen/core/Tensor.h>

namespace cfa {

// A strided GPU tensor whose memory the library can use as it is.  Callers let
// only torch.Tensor and Parameter themselves through, no other subclass.
inline bool plain(const at::Tensor &t) {
    return t.defined() && t.layout() == at::kStrided && t.is_cuda() && t.is_contiguous() && !t.is_conj() && !t.is_neg();
}

// Dtype codes; the first three as in the C ABI.
inline bool code_of(at::ScalarType t, int *code) {
    switch (t) {
    case at::kHalf: *code = 0; return true;
    case at::kBFloat16: *code = 1; return true;
    case at::kFloat: *code = 2; return true;
    case at::kChar: *code = 3; return true;
    case at::kLong: *code = 4; return true;
    default: return false;
    }
}

// A GPU tensor [.., C] whose last dimension is contiguous and whose others are
// n rows at one stride ld.
inline bool rows_view(const at::Tensor &t, int64_t *n, int64_t *C, int64_t *ld, int *code) {
    if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || t.is_conj() || t.is_neg() || t.dim() < 1 ||
        !code_of(t.scalar_type(), code))
        return false;
    const int64_t last = t.dim() - 1;
    *C = t.size(last);
    if (*C > 1 && t.stride(last) != 1)
        return false;
    int64_t stride = -1;
    *n = 1;
    for (int64_t d = last - 1; d >= 0; d--) {
        if (t.size(d) != 1) {
            if (stride < 0)
                stride = t.stride(d);
            else if (t.stride(d) != stride * *n)
                return false;
        }
        *n *= t.size(d);
        if (*n == 0)
            break;
    }
    *ld = stride < 0 || *n == 0 ? *C : stride;
    return true;
}

}  // namespace cfa
