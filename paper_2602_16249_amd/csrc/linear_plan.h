// Which tile a product takes and how its k is shared out, and what of a gradient's operands is copied (linear.hip): plain host code.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>

namespace affmae {
namespace {

constexpr int kCus = 256;

// Slices are 128 bytes of k deep: 64 values of bf16, 32 of fp32, two steps of one instruction of
// 32 of them / of four instructions of 4.
constexpr int kSliceBytes = 128;

// What a workgroup's tile costs, in us: a slice while a CU is full of such workgroups (per workgroup), a slice of one that has its CU
// to itself, and everything but the slices.  Measured on products of 16384 to 131072 rows, 64 to 2304 deep; large tiles read less of LDS
// per product (128 x 192 reaches 1.0 to 1.1 PFLOP/s in bf16), small ones fill the chip and hide their ends behind each other.
struct Shape {
  int bm, bn, resident;
  float slice, alone, end;
};
enum { k64x64, k128x64, k128x128, k128x192, kSlimTile };
constexpr Shape kForward16[] = {{64, 64, 4, .19f, .55f, .45f}, {128, 64, 4, .31f, .58f, 1.1f}, {128, 128, 4, .47f, .85f, 2.1f}, {128, 192, 3, .60f, 1.1f, 4.0f}, {16, 16, 4, .112f, .11f, .4f}};
constexpr Shape kGradient16[] = {{64, 64, 4, .183f, .55f, .57f}, {128, 64, 3, .283f, .58f, 1.2f}, {128, 128, 2, .546f, .85f, 2.2f}, {128, 192, 2, .70f, 1.1f, 3.7f}};
constexpr Shape kForward32[] = {{64, 64, 4, .66f, .78f, .4f}, {128, 64, 3, 1.17f, 1.22f, 1.4f}, {}, {}, {16, 16, 4, .116f, .11f, .4f}};
constexpr Shape kGradient32[] = {{64, 64, 4, .66f, 1.04f, .4f}, {128, 64, 3, 1.17f, 1.5f, 1.4f}, {}, {}};

struct Plan {
  int shape, splits;
};
// (floats: this is worked out for every call, several times)
float plan_cost(const Shape& h, float tiles, float values, uint32_t slices, uint32_t splits) {
  const float work = tiles * (float)splits, turn = (float)(kCus * h.resident), deep = (float)((slices + splits - 1) / splits);
  const float full = std::floor(work / turn), rest = std::ceil((work - full * turn) * (1.f / kCus));
  float t = full * (deep * std::max(h.alone, h.resident * h.slice) + h.resident * h.end);
  if (rest > 0.f) t += deep * std::max(h.alone, rest * h.slice) + rest * h.end;
  // parts are written and read once (4 TB/s), by one more launch
  if (splits > 1) t += 4.f + (float)splits * values * (8.f / 4e6f);
  return t;
}
// The cheapest tile; gradients also share a tile's k between workgroups: as many as make one or two full turns of the chip.
Plan plan_product(uint32_t M, uint32_t N, uint32_t K, int el, int line, bool forward) {
  const Shape* shapes = forward ? el == 2 ? kForward16 : kForward32 : el == 2 ? kGradient16 : kGradient32;
  const uint32_t deep = kSliceBytes / el, slices = (K + deep - 1) / deep;
  const float values = (float)M * (float)N;
  Plan best = {k64x64, 1};
  float least = 3e38f;
  for (int i = 0; i < (forward ? kSlimTile + 1 : kSlimTile); ++i) {
    const Shape& h = shapes[i];
    if (!h.bm || (i > k128x128 && line < 16)) continue;
    const float tiles = (float)((M + h.bm - 1) / h.bm) * (float)((N + h.bn - 1) / h.bn);
    if (i == kSlimTile && tiles > 1e6f) continue;
    for (int turns = 0; turns <= (forward ? 0 : 2); ++turns) {
      uint32_t splits = 1;
      if (turns) {
        const uint32_t most = (uint32_t)std::min((float)(kCus * h.resident * turns) / tiles, (float)(slices / 2));
        if (most < 2) continue;
        const uint32_t each = (slices + most - 1) / most;
        splits = (slices + each - 1) / each;  // (none without slices)
      }
      const float t = plan_cost(h, tiles, values, slices, splits);
      if (t < least) {
        least = t;
        best = {i, (int)splits};
      }
    }
  }
  return best;
}

int padded(int C, int el) { return (C * el + 15) / 16 * 16 / el; }

// What of the backward's operands is written anew, in rows of whole pieces.
struct Copies {
  bool dz, x, weight;
};
// dz with an activation or dropout anyway.  Else bf16 operands whose rows are no whole pieces, all or none, whichever gradients are asked for:
// with copies a product saves at least 4 us per 10^9 multiplications where rows are odd and 1 us where they are whole words, a copy costs 1.2 us
// per 10^6 values and its launch (dx and dW of 16384 x 767 -> 2303: 198 us instead of 498, of 16384 x 768 -> 2300 163 instead of 199; but
// 65536 x 255 -> 255, with copies of 34 million values, 109 instead of 99).
Copies copies(int rows, int Cin, int Cout, bool made, bool want_dx, bool want_dweight, int el) {
  const Copies c = {made, false, false};
  if (el == 4) return c;
  const bool in = Cin % 8, out = Cout % 8 && !made, odd = (in && Cin & 1) || (out && Cout & 1);
  const double macs = (double)rows * Cin * Cout, values = (out ? (double)rows * Cout : 0.) + (in ? ((double)rows + Cout) * Cin : 0.);
  if (!(in || out) || 2. * (odd ? 4e-9 : 1e-9) * macs <= 1.2e-6 * values + 8. * (out + 2 * in)) return c;
  return {made || out, in && want_dweight, in && want_dx};
}

}  // namespace
}  // namespace affmae
