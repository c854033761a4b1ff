// Launches of the paged cache's plan and write.
#include <algorithm>

#include "paged.hpp"
#include "seq_host.hpp"

namespace ma_host {

int run_paged_plan(Launcher &L, const ma::PagedPlan &p)
{
    // one slot a thread, up to a workgroup a compute unit
    const unsigned blocks = (unsigned)std::max<int64_t>(1, std::min<int64_t>(256, (p.capacity + 255) / 256));
    return L.run(kPagedPlan, [&] { return launched([&] { ma::paged_plan<<<dim3(blocks), dim3(256), 0, L.stream>>>(p); }); });
}

int run_paged_write(Launcher &L, const ma::PagedWrite &p)
{
    const int per = paged_write_rows(p.Hkv * p.d * p.size / 16);
    const unsigned blocks = (unsigned)(((int64_t)p.rows + per - 1) / per);
    return L.run(kPagedWrite, [&] { return launched([&] { ma::paged_write<<<dim3(blocks), dim3(256), 0, L.stream>>>(p, per); }); });
}

}  // namespace ma_host
