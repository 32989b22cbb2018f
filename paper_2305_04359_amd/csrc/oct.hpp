// 8-bit rows: what the kernels on them share.
#pragma once
#include "mx.hpp"

namespace annmi {

constexpr u32 OCT_STEP = 128;  // elements that share a scale: what one scaled matrix instruction takes of a row
constexpr u32 OCT_MOST_D = 1u << 20;
constexpr u64 OCT_MOST_ROWS = (1ull << 30) - 1;  // (their tiles are counted in workgroups, these in threads of 32 bits)

constexpr u32 oct_steps(u32 d) { return (d + OCT_STEP - 1) / OCT_STEP; }
constexpr u32 oct_words(u32 steps) { return (steps + 3) / 4; }  // of a row's scale bytes

// 8-bit rows as the kernels take them
struct OctRows {
  const uint8_t* codes;
  const uint32_t* scales;  // a byte for each step, whole words a row
  u32 n;
  u32 steps;
};

// the checks that all calls on 8-bit rows make of one set of them
int check_oct_rows(const char* what, const uint8_t* codes, const uint8_t* scales, u64 n, u32 d);

}  // namespace annmi
