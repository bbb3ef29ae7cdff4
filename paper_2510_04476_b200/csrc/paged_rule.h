// How attention over pages shares its units of rows out: by sizes and the device's room for clusters alone, and apart from the kernels, so that it
// compiles, and is checked, on a host without a device.
#pragma once

constexpr int PA_SIZES = 4;                 // clusters of 1, 2, 4 and 8 CTAs

// CTAs on the device at once, where n clusters of `size` of them find room; -1: such a cluster does not fit and must not be launched.
inline int cluster_ctas(int n, int size) { return n > 0 ? n * size : -1; }

// Ranks of a cluster that shares one (sequence, kv head), 0: the units are shared out over all CTAs and joined in a second launch.  The cheaper
// by a count of the units that follow one another: a CTA's own, as many times as there are turns of CTAs, or those that memory delivers in that
// time, whichever is more; 4 for a launch and 8 for two; and a 128th for each CTA in a cluster, which are started one after the other.
// runs: (sequence, kv head, pass) of the call; tiles: units of the longest sequence there may be; resident: CTAs that are on the device at once
// without clusters; room[i]: in clusters of 2^i, negative where such a cluster does not fit.
// Measured (us, caches of one length, clusters of 8 / the best smaller one / shared out), 8/2 x 128: 1 x 1024 4.4 / 5.5 / 5.9, 1 x 8192 14 / 25 / 8.0,
// 16 x 2048 7.3 / 8.3 / 11.8, 64 x 512 17 / 6.7 / 11.1, 256 x 2048 120 / 79 / 90; from memory 12 x 16384 35 / 41 / 39, 16 x 16384 43 / 48 / 49,
// 18 x 16384 (288 CTAs in clusters of 8 are more than find room) 61 / 52 / 53, 32 x 16384 83 / 80 / 85.
// The lengths are on the device: the rule takes the bound for every sequence.  Where one is long and the others are short, a cluster's CTAs work through the
// long one while the others have nothing left: one of 16384 rows and 31 (63) of 64 to 500 under that bound take 40 (74) us, the long one alone 10.
inline int paged_join_ranks(int dh, long long runs, long long tiles, long long resident, const int* room) {
  const long long flow = runs * tiles / (dh == 256 ? 80 : 160);             // (a unit is 64 KB at 256 channels, else 32 KB)
  auto larger = [](long long x, long long y) { return x > y ? x : y; };
  long long best = 128 * (8 + larger((runs * tiles + resident - 1) / resident, flow));
  int ranks = 0;
  for (int i = 0; i < PA_SIZES; ++i) {
    if (room[i] < 0) continue;
    const long long n = 1 << i, turns = (runs * n + room[i] - 1) / room[i];
    const long long cost = 128 * (4 + larger(turns * ((tiles + n - 1) / n), flow)) + (n > 1 ? runs * n : 0);
    if (cost < best) { best = cost; ranks = (int)n; }
  }
  return ranks;
}
