// Exact attention over sequences for element type float.
#include "seq_dispatch_fwd.hpp"

namespace ma_host {
template <> int run_seq_fwd<float>(Launcher &L, const ma::SeqFwd &p, const SeqPlan &how)
{
    return run_seq_fwd_impl<float>(L, p, how);
}
}  // namespace ma_host
