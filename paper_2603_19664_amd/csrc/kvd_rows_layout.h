// Launch geometry shared by the host code and kvd_rows.hip / kvd_evict.hip.
#pragma once

namespace kvd {

// Several query rows over stored keys (kvd_rows.hip).
constexpr int kRowsTile = 128;    // rows per workgroup of the tile kernel
constexpr int kRowsWave = 16;     // rows per workgroup of the fp32 kernel, all of them in each of its waves
constexpr int kRowsFew = 16;      // rows rows_few takes (one MFMA column block)
constexpr int kRowsTargetWgs = 512;
constexpr int kRowsLeastKeys = 128;  // keys per slot, at least (64: 1 % faster to 3 % slower, 256: 9 % faster to 7 % slower)
constexpr int kRowsSlotKeys = 512;   // a slot's fixed cost in keys
// rows whose states cost what a key costs a workgroup (48: up to 6 % slower, 192: up to 14 %)
constexpr int kRowsStateRows = 96;
constexpr int kRowsMostSlots = 64;
constexpr int kRowsSmall = 256;  // keys that one workgroup takes at once (512: up to 3 us slower)
// Waves that share a row's S states when they are merged: a wave keeps 8 in flight, so that
// many states are many round trips (512 rows of 66 states: 12.0 us with one wave per row, 9.2
// with four).
constexpr int rows_finish_waves(int S) { return S > 8 ? 4 : 1; }
// A launch has fewer than 2^32 threads.
constexpr long long most_wgs(int threads) { return ((1ll << 32) - 1) / threads; }

}  // namespace kvd
