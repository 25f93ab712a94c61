// Shared by the translation units of sp_attend.
#pragma once

#include "sp_common.h"
#include "sp_attend_plan.h"
#include "sp_score_internal.h"

namespace sp {

// Kernel-side view of sp_attend_args (passed by value).
struct AttendDev {
  int H, H_kv, G, T_new;
  int lg_page, blocks_per_seq;
  uint32_t last_page, last_row;  // of the pool, of a contiguous cache
  uint32_t most_items;           // (row, KV head) pairs to join that the list has room for
  float scale_log2;              // logit scale times log2(e)
  int64_t q_ts, q_hs, o_ts, o_hs;
  int32_t c_ts;                  // of the cache, in bytes
  int64_t c_hs, c_ps;
  uint64_t print;
  const AttendHeader* header;
  const AttendUnit* units;
  const AttendStretch* stretches;
  const AttendRow* rows;
  const int32_t* table;
  const uint16_t* q;
  const char* k;
  const char* v;
  const float* k_scale;
  const float* v_scale;
  uint16_t* out;
  float* lse;
  float* sums;                   // [slot][KV head][16][d]
  float2* stats;                 // [slot][KV head][16]: row maximum (of logits in log2 units), sum of weights
  const uint8_t* k_block_scale;  // of a 4-bit cache: the scale of the codes from byte x on is byte x / 16
  const uint8_t* v_block_scale;
  int heads_together;            // ... its rows are shorter than a cache line of 128 bytes, and those of a token's heads follow one another
};

sp_status check_attend_shape(const sp_attend_args* a);
sp_status check_attend_plan_args(const sp_attend_args* a);
void launch_attend_join(const AttendDev& p, int d, hipStream_t stream);

}  // namespace sp
