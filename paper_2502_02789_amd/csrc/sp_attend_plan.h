// How sp_attend cuts a call into pieces of work.  Plain C++: the kernel that makes the plan and a test without a GPU go
// through the same functions.
//
// The rows of a call are (token, head of a KV head's group) pairs, row = token * G + head, flat over all tokens: the rows of a
// sequence, and of a group of sequences, lie side by side.  A segment is a set of rows that attend to the same keys: the shared
// prefix of a group (all rows of its members), or what a sequence has for itself.  A segment is cut into blocks: one of 16 or 32 rows
// if it has no more (one or two small matrix tiles, bound by reading the keys), else of many_rows() (bound by the matrix cores).
//
// The device has room for attend_items() workgroups at once.  With fewer than three times as many (large block, KV head) pairs, blocks
// are laid end to end, each at its cost, and cut into as many stretches of equal cost as there is room for: every workgroup has one, and
// all end together.  With more than that a workgroup takes one block, and the device the next as one gets done, from the last sequence's last
// block to the first's first: longest first within a sequence, but sequences as they lie in the batch, whatever their lengths.  Only a
// block longer than a workgroup's equal share is cut.  Both measured, stretches against blocks: 64 sequences of 1K-4K keys 10 % less
// time, 64 that share 32K 5 %, two pieces of 500 tokens behind 17K 28 %; but, with more blocks than the rule allows, 6592 tokens of 64
// heads 23 % more, eight prompts of 300-3000 tokens, d = 64, 22 % more.
//
// A block of one piece whose rows have no shared prefix is finished by its workgroup; the pieces of all others leave their
// sums in slots of the workspace, which a second kernel joins.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "specprefill.h"

#ifdef __HIPCC__
#define SP_ATTEND_FN __host__ __device__ __forceinline__
#else
#define SP_ATTEND_FN inline
#endif

namespace sp {

constexpr int kTileRows = 16;     // rows of the smallest matrix tile
constexpr int kFewRows = 32;      // most rows of a block of a small segment: one such tile, or two
constexpr int kSlotRows = 16;     // rows of a workspace slot
constexpr int kShareRows = 128;   // see shares()
constexpr int kPieceStep = 64;    // pieces are cut at multiples of so many keys
constexpr int64_t kMostKeys = 0x7fff0000;  // of a cache, and of a sequence's room in one: indices some tiles further are 32-bit numbers still
constexpr int kMinSteps = 2;      // no piece is made shorter than so many steps
constexpr int kMostStretchBlocks = 3 * 768;  // blocks that stretches are made for, at most

// Waves of a workgroup, and the workgroups that the device has room for: one of eight waves on each of 256 compute units, or, as
// d = 64 takes a quarter of the LDS and fewer registers, three of four
SP_ATTEND_FN constexpr int attend_waves(int d) { return d == 64 ? 4 : 8; }
SP_ATTEND_FN constexpr int attend_items(int d) { return d == 64 ? 768 : 256; }
// Rows of a block that has more than 32: 32 for each wave
SP_ATTEND_FN constexpr int many_rows(int d) { return 32 * attend_waves(d); }

struct AttendUnit {   // one piece of one block
  int32_t r0, nr;     // first row, rows (nr <= 32: the kernel part for few rows)
  int32_t seq;        // whose block table is read; of a contiguous cache: the row of its first token
  int32_t k0, k1;     // keys [k0, k1)
  int32_t off;        // token t sees keys below t + off (kNoLimit: all of the piece)
  int32_t slot;       // where the sums go, or -1: the block is finished here
  int32_t run;        // kBadUnit: the sequence's length is invalid, its rows become NaN; else how many units from this one on are taken side by side (0: this one alone)
};
struct AttendStretch {  // what one workgroup does, for each KV head: units [first, end), the first of them a copy
  int32_t first, end;
  int32_t pad[2];
  AttendUnit unit;
};
struct AttendJoin {   // one block of a sequence's own rows that slots are joined for
  int32_t r0, nr;
  int32_t own_slot, own_pieces, own_step;           // slot of the first piece, pieces, slots of a piece
  int32_t first;                                    // its first row among all that are joined
  int32_t group;                                    // whose prefix the rows have as well, or -1
  int32_t pad;
};
struct AttendRow {    // one of these rows: where its sums are, slot * 16 + row of the slot (KV heads aside), and how far apart
  int32_t row;
  int32_t own_at, own_pieces, own_step;
  int32_t pre_at, pre_pieces, pre_step;
  int32_t pad;
};
struct AttendHeader {
  uint64_t print;     // of the shape fields the plan was made for
  int32_t n_stretches, n_rows;  // workgroups for each KV head, rows to join
  int32_t most_pieces;      // of a row to join
  int32_t pad;
};

constexpr int kNoLimit = 0x7fffffff;
constexpr int kBadUnit = -1;

struct AttendCaps {
  int64_t blocks, units, joins, rows, slots;
};

// Upper bounds for any lengths that the shape fields allow.  Blocks: a segment of R rows has at most R / many_rows() + 1; own segments
// with a block: at most B and at most one per row; prefix segments: n_groups.  Pieces: cuts add at most attend_items() / H_kv to one per block.
// Slots: prefix blocks, blocks of sequences with a prefix, and blocks of several pieces, of which there are at most as many as pieces added; a
// prefix is only shared where a group has fewer than 128 rows per member on average (shares()), so rows in such groups are fewer than 128 B.
inline AttendCaps attend_caps(const sp_attend_args* a) {
  const int64_t many = many_rows(a->d), rows = a->T_new * (a->H / a->H_kv), added = attend_items(a->d) / a->H_kv + 1;
  const int64_t own_segments = rows < a->B ? rows : a->B, own = rows / many + own_segments;
  const int64_t shared_rows = rows < (int64_t)kShareRows * a->B ? rows : (int64_t)kShareRows * a->B;
  const int64_t groups = a->n_groups < own_segments ? a->n_groups : own_segments;  // those with a row
  const int64_t prefix = a->n_groups ? shared_rows / many + groups : 0;
  AttendCaps c;
  c.blocks = own + prefix;
  c.units = c.blocks + added;
  c.joins = own;
  // rows to join: of blocks that are cut (of which there are at most as many as pieces added) and of sequences that share
  const int64_t cut_rows = many * added + (a->n_groups ? shared_rows : 0);
  c.rows = rows < cut_rows ? rows : cut_rows;
  // blocks that may leave sums, in large blocks and in all; segments of over 16 (32) rows: at most one per 17 (33)
  const int64_t per_big = rows / (kFewRows + 1), per_two = rows / (kTileRows + 1);
  const int64_t shared_big = a->n_groups ? 2 * (shared_rows / many) + (own_segments < per_big ? own_segments : per_big) + (groups < per_big ? groups : per_big) : 0;
  const int64_t shared_few = a->n_groups ? own_segments + groups + (own_segments < per_two ? own_segments : per_two) + (groups < per_two ? groups : per_two) : 0;
  // pieces of blocks that are cut: at most two for each piece added
  c.slots = (rows > kFewRows ? many / kSlotRows : rows > kTileRows ? 2 : 1) * (2 * added) + (many / kSlotRows) * shared_big + shared_few;
  return c;
}

// The most rows that a group may share a prefix with, 128 for each member on average: a block's rows are filled up by several members, and
// its keys read once for them all; with 128 rows of its own for each member there is little to gain.  (prefix_pays() asks for more.)
SP_ATTEND_FN bool shares(int rows, int members) { return members >= 2 && rows / kShareRows < members; }

// (Rows of a segment are fewer than 2^31: T_new * H is.  Divisions of 64-bit numbers take 150 instructions each; the plan, one workgroup that
// goes through its code once, is bound by fetching it.)
SP_ATTEND_FN int block_rows(int rows, int d) { return rows <= kTileRows ? kTileRows : rows <= kFewRows ? kFewRows : many_rows(d); }
SP_ATTEND_FN int segment_blocks(int rows, int d) {
  const uint32_t m = (uint32_t)block_rows(rows, d);
  const int shift = m == 16 ? 4 : m == 32 ? 5 : m == 128 ? 7 : 8;
  return (int)(((uint32_t)rows + m - 1) >> shift);
}

// One past the last key that row `row` of a sequence sees (its rows counted from 0, G to a token), n new tokens, len keys.
SP_ATTEND_FN int row_limit(uint32_t row, int G, int n, int len) {
  const int64_t v = (int64_t)len - n + row / (uint32_t)G + 1;
  return v < 0 ? 0 : v > len ? len : (int)v;
}

// The keys of block i (of m rows) of a sequence's own segment: [shared, the limit of its last row)
SP_ATTEND_FN int own_block_keys(int rows, int i, int m, int G, int n, int len, int shared) {
  const uint32_t end = (uint32_t)(i + 1) * (uint32_t)m, last = (end < (uint32_t)rows ? end : (uint32_t)rows) - 1;
  const int v = row_limit(last, G, n, len) - shared;
  return v < 0 ? 0 : v;
}

// Steps of 64 keys of a block's keys [first, first + keys), cut at multiples of 64 keys of the sequence
SP_ATTEND_FN int block_steps(int first, int keys) { return (int)(((uint32_t)(first & (kPieceStep - 1)) + (uint32_t)keys + kPieceStep - 1) / kPieceStep); }

// A piece of few rows and few keys is not worth all waves: where several follow one another, they share the waves.  (64 sequences of
// 200-1000 keys take 7 % less time so; up to 4096 keys instead of 1024: the same, but 64 that share 32K 1.5 % more.)
SP_ATTEND_FN bool is_short(int rows, int keys) { return rows <= kFewRows && keys <= 1024; }

// What a step costs a workgroup, in units of 0.27 us (d = 128) and 0.67 us on a full device: few rows are bound by reading 64 keys
// and values, more by the matrix cores; and what a piece costs besides.  (Few and many rows alike: 24 sequences of 1 to 8 new tokens
// that share 8K 4 % slower, two pieces of 500 tokens behind 17K 2 %; large blocks alike, however many
// of their rows are there: 32 sequences that share 32K 8-bit keys 11 %.)
SP_ATTEND_FN int step_cost(int rows, int d, bool fp8) {
  if (rows <= kTileRows) return d == 64 ? (fp8 ? 2 : 3) : (fp8 ? 3 : 5);
  if (rows <= kFewRows) return d == 64 ? 4 : fp8 ? 4 : 6;
  return d == 64 ? 4 : rows > many_rows(d) / 2 ? 8 : fp8 ? 5 : 6;
}
SP_ATTEND_FN int piece_cost(int rows, int keys, int d) { return d == 64 ? (is_short(rows, keys) ? 2 : 4) : is_short(rows, keys) ? 3 : 12; }
// No stretch costs less: more than a step of any kind.  (Three times as much: one token behind 1000 keys 4 % slower, 64 that share
// 32K 2 %.)
SP_ATTEND_FN int least_stretch(int d) { return d == 64 ? 10 : 11; }

// Whether `members` sequences with `rows` rows in all, about as many each, have the `prefix` tokens that they share read once for all of them.
// Without that each reads them, the first at a step's cost and the others out of the caches, at 2 a step for one tile of rows, 3 for two and 5
// for more.  With it the rows' blocks read them once, but every row of every member leaves its sums to the join, which with what its
// prefix's block costs besides comes to 5/4 a row.  (A step is 64 keys.)  Measured
// (read by each, once for all): 64 sequences, 1000 keys of their own, four heads: 64 shared tokens 47.7, 50.4 us, 512 54.8, 49.9, 4096 113,
// 55.7; four new tokens each: 64 48.9, 68.0, 512 55.6, 64.9, 2048 76.7, 63.6; 24 sequences of 8 tokens of eight heads: 512 41.3, 44.5,
// 4096 86.1, 66.8; two of one token: 4096 12.7, 12.4.  Over 2456 such calls the rule loses 1.8 % against the better of the two (at worst 1.5
// times; against sharing always 1.3), sharing always 8.6 % (at worst 2.6 times), never 19 %.
SP_ATTEND_FN bool prefix_pays(int rows, int members, int prefix, int d, bool fp8) {
  if (prefix <= 0 || !shares(rows, members)) return false;
  const int own = (int)((uint32_t)rows / (uint32_t)members), many = many_rows(d), whole = rows > kFewRows ? (int)((uint32_t)rows / (uint32_t)many) : 0;
  const int rest = rows - whole * many;
  const int64_t each = step_cost(own, d, fp8) + (int64_t)(members - 1) * (own <= kTileRows ? 2 : own <= kFewRows ? 3 : 5);
  const int64_t once = (int64_t)whole * step_cost(many, d, fp8) + (rest > 0 ? step_cost(rest, d, fp8) : 0);
  return prefix * (each - once) >= (int64_t)rows * (kPieceStep * 5 / 4);
}

// many: blocks of more than 32 rows (the others are cheap to cut)
SP_ATTEND_FN bool by_stretches(int64_t blocks, int64_t many, int d, int H_kv) {
  return many * H_kv < 3 * (int64_t)attend_items(d) && blocks <= kMostStretchBlocks;
}
// Stretches for each KV head, blocks of `cost` in all: what the device has room for, as long as that leaves each enough to do
SP_ATTEND_FN int stretch_count(int64_t cost, int d, int H_kv) {
  const int64_t room = attend_items(d) / H_kv > 0 ? attend_items(d) / H_kv : 1, most = cost / least_stretch(d);
  return (int)(most < 1 ? 1 : most < room ? most : room);
}
// Most workgroups for each KV head that any lengths can give: of stretches where there cannot be too many blocks for them, and
// no more than the longest sequences that the cache has room for ask for
inline int64_t most_stretches(const sp_attend_args* a) {
  const AttendCaps c = attend_caps(a);
  const int64_t rows = a->T_new * (a->H / a->H_kv);
  const int64_t large = rows > kFewRows ? c.blocks : 0;
  if (!by_stretches(c.blocks, large, a->d, a->H_kv)) return c.units;
  const int64_t room = a->d_block_table ? (int64_t)a->blocks_per_seq * a->page_size : a->n_rows;
  const int64_t steps = room / kPieceStep + 2, step = a->d == 64 ? 4 : large ? 8 : 6, extra = 12;
  return stretch_count(c.blocks * (steps * step + extra), a->d, a->H_kv);
}
// Where stretch s of n begins, blocks laid end to end (exact: products are below 2^53, and quotients far enough from whole numbers)
SP_ATTEND_FN int64_t stretch_start(int64_t cost, int n, int s) { return (int64_t)((double)cost * s / n); }
// ... as a step of the block whose share begins at `start` (what the block costs besides spread over its steps): `steps` (the next
// block's first) or 0 where a piece would get too short.  Does not descend as x ascends.
SP_ATTEND_FN int step_at(int64_t x, int64_t start, int steps, int per_step, int extra) {
  const double cost = (double)steps * per_step + extra;
  const int j = (int)((double)(x - start) * steps / cost + 0.5);
  return j < kMinSteps ? 0 : steps - j < kMinSteps ? steps : j;
}
SP_ATTEND_FN int step_key(int first, int keys, int steps, int j) {
  return j <= 0 ? first : j >= steps ? first + keys : (first & ~(kPieceStep - 1)) + j * kPieceStep;
}

// Otherwise: most keys of a piece, for `total` keys summed over all blocks
SP_ATTEND_FN int make_cut(int64_t total, int d, int H_kv) {
  const int items = attend_items(d) / H_kv > 0 ? attend_items(d) / H_kv : 1;
  const int64_t share = (total + items - 1) / items, least = kMinSteps * kPieceStep;
  const int64_t cut = (share + kPieceStep - 1) / kPieceStep * kPieceStep;
  return cut < least ? (int)least : cut > 0x40000000 ? 0x40000000 : (int)cut;
}
SP_ATTEND_FN int pieces_of(int keys, int cut) { return keys <= cut ? 1 : (int)(((uint32_t)keys + (uint32_t)cut - 1) / (uint32_t)cut); }
// first step of piece p of so many (exact, as above)
SP_ATTEND_FN int piece_step(int steps, int pieces, int p) { return (int)((double)steps * p / pieces); }
// first key of piece p
SP_ATTEND_FN int piece_start(int first, int keys, int pieces, int p) {
  const int steps = block_steps(first, keys);
  return step_key(first, keys, steps, p == pieces ? steps : piece_step(steps, pieces, p));
}

SP_ATTEND_FN uint64_t attend_print(const sp_attend_args* a) {
  const uint64_t v[] = {0x61747465ull, (uint64_t)(uint32_t)a->B, (uint64_t)(uint32_t)a->H, (uint64_t)(uint32_t)a->H_kv, (uint64_t)(uint32_t)a->d,
                        (uint64_t)a->T_new, (uint64_t)(uint32_t)a->n_groups, a->d_block_table ? (uint64_t)(uint32_t)a->page_size : 0,
                        a->d_block_table ? (uint64_t)(uint32_t)a->blocks_per_seq : 0, (uint64_t)a->n_rows, (uint64_t)(uint32_t)a->cache_dtype};
  uint64_t h = 1469598103934665603ull;  // each field mixed in by a product and a shift
  for (uint64_t x : v) {
    h = (h ^ x) * 0x9E3779B97F4A7C15ull;
    h ^= h >> 29;
  }
  return h | 1;  // never zero: cleared memory is no plan
}

// Offsets of the parts of d_plan
struct AttendPlanLayout {
  size_t units, stretches, joins, rows, seg_start, seqs, groups, bytes;
};
inline size_t attend_round(size_t x) { return (x + 255) / 256 * 256; }
inline AttendPlanLayout attend_plan_layout(const sp_attend_args* a) {
  const AttendCaps c = attend_caps(a);
  AttendPlanLayout l;
  size_t at = 256;
  l.units = at; at += attend_round(sizeof(AttendUnit) * (size_t)c.units);
  l.stretches = at; at += attend_round(sizeof(AttendStretch) * (size_t)c.units);
  l.joins = at; at += attend_round(sizeof(AttendJoin) * (size_t)c.joins);
  l.rows = at; at += attend_round(sizeof(AttendRow) * (size_t)c.rows);
  l.seg_start = at; at += attend_round(4 * ((size_t)a->B + (size_t)a->n_groups + 1));
  l.seqs = at; at += attend_round(16 * (size_t)a->B);
  l.groups = at; at += attend_round(32 * (size_t)a->n_groups);
  l.bytes = at;
  return l;
}
// Workspace: sums fp32 [slot][KV head][16 rows][d], then (maximum, sum of weights) [slot][KV head][16 rows]
inline size_t attend_sums_bytes(const sp_attend_args* a) {
  return attend_round((size_t)attend_caps(a).slots * (size_t)a->H_kv * kSlotRows * (size_t)a->d * 4);
}
inline size_t attend_workspace(const sp_attend_args* a) {
  return attend_sums_bytes(a) + attend_round((size_t)attend_caps(a).slots * (size_t)a->H_kv * kSlotRows * 8);
}

}  // namespace sp
