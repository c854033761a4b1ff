// The gradient of exact attention over packed sequences for element type _Float16.
#include "seq_dispatch_bwd.hpp"

namespace ma_host {
template <> int run_seq_bwd<_Float16>(Launcher &L, const ma::SeqBwd &p) { return run_seq_bwd_impl<_Float16>(L, p); }
}  // namespace ma_host
