// The gradient of exact attention over packed sequences for element type __bf16.
#include "seq_dispatch_bwd.hpp"

namespace ma_host {
template <> int run_seq_bwd<__bf16>(Launcher &L, const ma::SeqBwd &p) { return run_seq_bwd_impl<__bf16>(L, p); }
}  // namespace ma_host
