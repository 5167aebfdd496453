// The host-side rules of the paged attention's launch, for tests/test_paged_host.py.
#include "../../paper_2501_08071_amd/csrc/attn_paged_launch.h"

extern "C" int divided(int n, int d) { return Divisor(d).of(n); }
// rows, workgroups, balanced, direct, waves, prefix_rows, prefix_tiles, prefix_splits, bytes
extern "C" void plan(int B, int T, int Hq, int Hk, int D, int max_q, int max_kv, int prefix_len, long long* out) {
    const PagedPlan p = paged_plan(B, T, Hq, Hk, D, max_q, max_kv, prefix_len);
    const long long v[] = {p.rows, p.workgroups, p.balanced, p.direct, p.waves, p.prefix_rows, p.prefix_tiles, p.prefix_splits, p.bytes, p.part_floats, p.prefix_floats};
    for (int i = 0; i < 11; ++i) out[i] = v[i];
}
extern "C" long long key_offset(int j, int mask, int row_bytes) { return (long long)paged_key_offset(j, mask, row_bytes); }
