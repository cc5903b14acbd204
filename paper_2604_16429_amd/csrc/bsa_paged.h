// Attention over a cache in pages: what its kernels share.
//
// Sequence b has P tokens that all sequences share (the prefix), then kl of its own; its ql queries
// stand at its end.  Query i is token p = P + kl - ql + i and sees token j where
//   j <= p  and  (j >= p - left or j < sinks).
// The query heads that share a key/value head are rows of one problem, as in the windowed attention:
// row r of a (sequence, key/value head) slice is query token r / group, head r % group.
#pragma once

#include "bsa_paged_plan.h"
#include "bsa_window.h"

namespace bsa {

namespace paged {

using win::kLn2;
using win::kLog2e;
using win::kNoRef;
using win::put4;

// The same for all lanes, in scalar registers.
__device__ __forceinline__ int prefix_of(const Shape& s)
{
    const int p = s.prefix_len ? min(max(*s.prefix_len, 0), s.prefix_tokens) : s.prefix_tokens;
    return __builtin_amdgcn_readfirstlane(p);
}
__device__ __forceinline__ Sequence sequence(const Shape& s, int b)
{
    Sequence q;
    q.ql = __builtin_amdgcn_readfirstlane(s.q_lens ? min(max(s.q_lens[b], 0), s.q_tokens) : s.q_tokens);
    q.kl = __builtin_amdgcn_readfirstlane(min(max(s.k_lens[b], 0), s.table_pages << s.page_shift));
    q.prefix = prefix_of(s);
    return q;
}

}  // namespace paged

hipError_t launch_paged_fwd(bool is_bf16, int D, const paged::Shape& s, const void* q, const void* k,
                            const void* v, void* out, float* lse, void* workspace,
                            hipStream_t stream);
size_t paged_fwd_workspace(bool is_bf16, int D, const paged::Shape& s);

}  // namespace bsa
