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
