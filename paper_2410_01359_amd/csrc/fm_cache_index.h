// Where tokens lie in the paged cache, which keys a sequence's rows can see, and how those are cut into chunks.  Index values
// come from the caller's device memory: nothing here follows one out of its range.  Plain integer code: the host compiles it too.
#pragma once
#include "fm_direct_order.h"

// Keys are counted in groups of 16: pages hold whole groups.
constexpr int FM_KEY_GROUP = 16;
// The page that a table entry names, -1: none.
FM_HOST_DEVICE inline int fm_known_page(int entry, int num_pages) { return entry >= 0 && entry < num_pages ? entry : -1; }

// Place of a token: column of its sequence's row and slot in the page; column = -1 where the table has none.
struct FmPlace {
  int column, slot;
};
FM_HOST_DEVICE inline FmPlace fm_place(int position, const FmDivisor& page, int columns) {
  if (position < 0) return FmPlace{-1, 0};
  const int column = fm_div(position, page);
  return FmPlace{column < columns ? column : -1, position - column * (int)page.n};
}

// Keys of a sequence of `len` tokens that any of its last T rows can see, bounds apart: [lo, hi) with lo a multiple of
// FM_KEY_GROUP and hi within the table; len is held to 0 from below.
struct FmKeyRange {
  int len, lo, hi;
};
FM_HOST_DEVICE inline FmKeyRange fm_key_range(int len, int T, int window, int table_keys) {
  FmKeyRange r;
  r.len = len > 0 ? len : 0;
  r.hi = r.len < table_keys ? r.len : table_keys;
  r.lo = 0;
  if (window > 0) {
    const long long first = (long long)r.len - T + 1 - window;   // of the first row
    if (first > 0) r.lo = (int)(first / FM_KEY_GROUP * FM_KEY_GROUP);
  }
  if (r.lo >= r.hi) r.lo = r.hi = 0;
  return r;
}
FM_HOST_DEVICE inline int fm_key_groups(const FmKeyRange& r) { return (r.hi - r.lo + FM_KEY_GROUP - 1) / FM_KEY_GROUP; }

// Rows of [lo, hi) that are neither in [lts, lte) nor in [uts, ute).  Bounds are any numbers of 32 bits, such as an end far below its start for an empty
// interval: they are held to the rows first, so that no difference is larger than hi - lo, which the caller keeps within 32 bits.
FM_HOST_DEVICE inline int fm_rows_left(int lo, int hi, int lts, int lte, int uts, int ute) {
  if (lo >= hi) return 0;
  const auto held = [=](int i) { return i < lo ? lo : i > hi ? hi : i; };
  const int a0 = held(lts), b0 = held(lte), a1 = held(uts), b1 = held(ute);
  const int first = b0 > a0 ? b0 - a0 : 0, second = b1 > a1 ? b1 - a1 : 0;
  const int begin = a0 > a1 ? a0 : a1, end = b0 < b1 ? b0 : b1;   // of what both have
  return hi - lo - first - second + (end > begin ? end - begin : 0);
}

// Groups of a chunk where sequences of `total` groups together are meant to be cut into `chunks`: a multiple of `round`, at least `least`.
FM_HOST_DEVICE inline int fm_chunk_groups(unsigned total, const FmDivisor& chunks, int least, int round) {
  unsigned size = fm_div((int)(total + chunks.n - 1), chunks);
  if (size < (unsigned)least) size = least;
  return (int)((size + round - 1) / round * round);
}
// Chunks of a sequence: at least one, so that somebody writes an empty sequence's rows.
FM_HOST_DEVICE inline int fm_chunks_of(int groups, int size) { return groups > size ? (groups + size - 1) / size : 1; }
// Groups of each of a sequence's chunks: as equal as multiples of `round` are (a last chunk may be empty), no more than the size they
// were counted with where that is a multiple of `round`, too.
FM_HOST_DEVICE inline int fm_even_chunk(int groups, int chunks, int round) {
  return (int)(((unsigned)(groups + chunks - 1) / (unsigned)chunks + round - 1) / round * round);
}
// Where the panel behind the one at `panel` begins: panels have `keys` keys, or 0: one has everything up to `end`.
FM_HOST_DEVICE inline int fm_next_panel(int panel, int end, int keys) { return keys > 0 && end - panel > keys ? panel + keys : end; }
// Chunks of all sequences together and partial results that they leave, at most: a sequence of several chunks has fewer than
// twice its groups / size, and any has fewer than that and one.
FM_HOST_DEVICE inline int fm_most_units(int chunks, int sequences) { return chunks + sequences; }
FM_HOST_DEVICE inline int fm_most_slots(int chunks, int sequences) { return chunks < sequences ? 2 * chunks : chunks + sequences; }

// Sequences of tables up to this many keys are not split: one launch.  round, least: groups that the waves of a team take in a step, and of a
// chunk at least; workgroups: of such a call.  What cannot be split goes whole; a splitting call's second launch and longer way to
// its first keys cost about three steps, and the more the fuller the chip is; a table says how long sequences may be, not how long they
// are, so that 1024 keys are the most.  Steps of 64 keys (two teams of 32 query rows) count as 128, of 512 (d = 64, 8 bits) as 256.
// us whole / split, 8 K/V heads, d = 128, 16 bits (step 128): one sequence of 384 / 512 / 640 keys 8.7/9.9, 9.8/9.8, 10.8/9.9; 16 of 768
// 14.1/17.6, of up to 768 12.9/13.3, of up to 1280 18.3/17.4; 64 of 1024 44.8/47.4.  One sequence, d = 64 (step 256), 768 / 1024 keys 9.9/10.8,
// 11.4/10.8; 8 bits 11.6/12.3, 11.7/12.6, of 1280 14.4/12.6.  Over 1068 such points calls take 0.2 % more than on the better side of each.
FM_HOST_DEVICE inline long long fm_whole_keys(int round, long long workgroups, int least, int cus) {
  long long keys = round * FM_KEY_GROUP;
  keys = keys < 128 ? 128 : keys > 256 ? 256 : keys;
  keys *= 3 + 6 * workgroups / (cus > 0 ? cus : 256);
  if (keys > 1024) keys = 1024;
  return keys > (long long)least * FM_KEY_GROUP ? keys : (long long)least * FM_KEY_GROUP;
}
// Whether trees of T tokens with `rows` query rows to a K/V head go through tree_kernel, which reads keys and values once for 128 rows, or decode_kernel, which has
// room for 64 tokens.  8-bit values of 128 elements cost the first more to widen than they save until there are more rows.  us, decode_kernel / tree_kernel, at 32, 48,
// 64, 80, 128 and 252 rows: 16 trees over ragged caches of up to 8192 keys, 8 K/V heads, d = 128, 16 bits 50/49 61/52 64/53 81/56 108/63 159/105, 8 bits
// 38/51 53/58 56/59 70/62 87/70 132/123, d = 64 36/31 45/38 47/38 60/40 77/43 111/70, 8 bits 32/32 42/39 45/39 57/41 73/45 104/73; one over 8192 19/21 21/24
// 24/24 26/26 34/32 55/36; 64 over up to 1500 47/51 60/55 64/56 80/59 95/68 127/111, 8 bits 38/58 53/61 57/62 72/65 83/74 103/130.  Over 504 such points calls take
// 1.4 % more than on the better side of each (from 64 rows on whatever the type: 2.8 %), at most 1.4 times as much: 100 over up to 500 keys, 2 K/V heads, 8 bits
// 13/26 18/27 19/29 24/29 22/31 36/36.
FM_HOST_DEVICE constexpr bool fm_tree_is_wide(long long rows, int T, int d, bool e4m3) { return T > 63 || rows >= (e4m3 && d == 128 ? 80 : 48); }

// Which of two joins a call on trees takes behind its chunks: true: a few lanes to a row, all of a sequence's chunks one behind the other
// (tree_join_kernel); false: a workgroup to a row, chunks side by side (join_kernel).  rows: of all heads; chunks: that all sequences are meant to be cut into;
// keys: of a row of the table.  The first takes as long as the longest sequence has chunks, 0.15 us each; the other 0.35 us for every 1000
// rows of all sequences.  The longest is taken to have four times its share.  us, join_kernel / tree_join_kernel, d = 128: 16 sequences of up to
// 8192 keys, 2016 rows, 32 chunks 16.2/6.2, 128 rows, 256 chunks 5.1/11.0; one, 2016 rows 7.8/9.4, 512 rows, 64 chunks 4.9/15.6, 8064 rows, 8 chunks
// 10.0/7.3; four of 2000, 2016 rows, 32 chunks 10.2/6.8; 64 of up to 1500, 2016 rows, 64 chunks 44/10, 128 rows, 256 chunks 7.2/4.6.
FM_HOST_DEVICE inline bool fm_tree_joins_by_lanes(long long rows, int sequences, int chunks, int least, long long keys) {
  long long longest = (4ll * chunks + sequences - 1) / sequences;
  if (longest > chunks) longest = chunks;
  const long long most = (keys + least * FM_KEY_GROUP - 1) / (least * FM_KEY_GROUP);
  if (longest > most) longest = most;
  return rows * sequences >= 200 * longest;
}
// Split sequences at most: each has two partial results at least.  Units of a launch: those above, in whole rounds of the XCDs.
FM_HOST_DEVICE inline int fm_most_splits(int chunks, int sequences) { return chunks < sequences ? chunks : sequences; }
FM_HOST_DEVICE inline int fm_listed_units(int chunks, int sequences) { return (fm_most_units(chunks, sequences) + 7) / 8 * 8; }

// Row of a fork's child: what its column c holds.  `entry`: the parent's, -1 without a known parent.
struct FmFork {
  int last;      // column of the last page
  bool partly;   // it is neither full nor empty
};
FM_HOST_DEVICE inline FmFork fm_fork(int len, const FmDivisor& page) {
  FmFork f = {0, false};
  if (len > 0) {
    f.last = fm_div(len, page);
    f.partly = len != f.last * (int)page.n;
  }
  return f;
}
FM_HOST_DEVICE inline int fm_fork_entry(const FmFork& f, int c, int entry, int fresh) {
  if (fresh < 0 || c < f.last) return entry;
  return c == f.last && f.partly ? fresh : -1;
}
