// The gradient of exact attention over packed sequences for element type float.
#include "seq_dispatch_bwd.hpp"

namespace ma_host {
template <> int run_seq_bwd<float>(Launcher &L, const ma::SeqBwd &p) { return run_seq_bwd_impl<float>(L, p); }
}  // namespace ma_host
