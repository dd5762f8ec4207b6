// The plan of an attention call in libgrkv.so as plain numbers, for
// tests/test_host_serving.py (no GPU work).
#include "grkv_internal.h"

// out: rt, row groups, splits, min_tiles, rows, tile_keys, grouped, joined, even, blocks, opart, mpart, flags, total
extern "C" void attend_probe(int32_t entries, int32_t group, int32_t tokens, int32_t d, int32_t dtype, int64_t slots,
                             int32_t ragged, int64_t* out) {
  const grkv::AttendPlan p = grkv::attend_plan(entries, group, tokens, d, dtype, slots, ragged != 0);
  const int64_t v[14] = {p.rt, p.row_groups, p.splits, p.min_tiles, p.rows, p.tile_keys, p.grouped, p.joined, p.even,
                         p.blocks, (int64_t)p.opart, (int64_t)p.mpart, (int64_t)p.flags, (int64_t)p.total};
  for (int i = 0; i < 14; ++i) out[i] = v[i];
}
