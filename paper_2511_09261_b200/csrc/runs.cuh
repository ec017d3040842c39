// Runs of rows whose weight gradients are summed apart (host side).
#pragma once

#include <stdint.h>

#include <vector>

constexpr int kWgChunkMinRows = 2048; // a subgraph is split for the weight gradient only in runs at least this long

// One accumulator of the tensor core takes no more rows than this: it cuts off what does not fit when it adds 16 rows, up to 2^-23 of
// the accumulator each time (4,096 times here: 5e-4 at most, in bfloat16 features less than the stored dg's 2^-8; a million rows in
// one run would lose 1 %).  The gated feed-forward block keeps to it.
constexpr int64_t kMostRunRows = 65536;

// rows of a run that give every SM some four of them
inline int64_t run_rows(int64_t n, int sm_count) {
  const int64_t sms = sm_count > 0 ? sm_count : 148;
  const int64_t per = (n + 4 * sms - 1) / (4 * sms);
  const int64_t rows = (per + 63) / 64 * 64;
  return rows < kWgChunkMinRows ? kWgChunkMinRows : rows;
}

// Begin, end and slot of every run, in order (slot >= 0: of partial sums; -(s + 1): subgraph s is one run), and of every split subgraph its
// number, first slot and count of slots.
struct HostRuns {
  std::vector<int32_t> wb, we, wsl, mp, mf, mc;
  int32_t n_wg_slots = 0;
};

// The subgraphs with active[s] != 0 (nullptr: all) in runs of at most `rows` rows.  Slots are numbered over ALL subgraphs.
inline void cut_runs(const std::vector<int32_t>& part_ptr, int32_t S, int64_t rows, const uint8_t* active, HostRuns& o) {
  int32_t slots = 0;
  for (int32_t s = 0; s < S; ++s) {
    const int32_t a = part_ptr[s], b = part_ptr[s + 1];
    const bool on = !active || active[s];
    const int32_t first_slot = slots;
    if (b - a <= rows) {
      if (on) {
        o.wb.push_back(a);
        o.we.push_back(b);
        o.wsl.push_back(-(s + 1));
      }
      continue;
    }
    slots += (int32_t)((b - a + rows - 1) / rows);
    if (!on) continue;
    for (int64_t r = a, k = 0; r < b; r += rows, ++k) {
      o.wb.push_back((int32_t)r);
      o.we.push_back((int32_t)(r + rows < b ? r + rows : b));
      o.wsl.push_back(first_slot + (int32_t)k);
    }
    o.mp.push_back(s);
    o.mf.push_back(first_slot);
    o.mc.push_back(slots - first_slot);
  }
  o.n_wg_slots = slots;
}
