// Exact attention over sequences for element type __bf16.
#include "seq_dispatch_fwd.hpp"

namespace ma_host {
template <> int run_seq_fwd<__bf16>(Launcher &L, const ma::SeqFwd &p, const SeqPlan &how)
{
    return run_seq_fwd_impl<__bf16>(L, p, how);
}
}  // namespace ma_host
