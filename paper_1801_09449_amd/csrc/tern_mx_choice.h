// The launch of a product on block-scaled numbers (tern_mx_product.hip), chosen from sizes alone.  Host code without
// HIP, so that a test can compile it by itself.
#pragma once
#include <stdint.h>

namespace tern {

// Kernels: direct ones, whose waves take a share of k each straight from memory and add up at the end, with 1 x 1 or
// 2 x 2 blocks of 32 x 32 to a workgroup, and tiled ones with 4 x 4 or 8 x 8.  And, for gradients, one that takes its wide
// side from its source (tern_mx_narrow.hip), where the other has at most kNarrowRows rows (kNarrowInputs: A's, against a B in
// parts).
enum ProductForm { kDirect1 = 0, kDirect2 = 1, kTiled4 = 2, kTiled8 = 3, kForms = 4, kNarrow = kForms };
enum WideSide { kWideNone = 0, kWideDyRows, kWideDyDown, kWideWeights, kWideInput };
constexpr int kMostSplits = 64, kNarrowRows = 64, kNarrowInputs = 128;

struct ProductSize {
    int64_t na, nb;                 // output extents
    int64_t groups, parts;          // records of a row block, and how many operands B comes in
};
struct ProductPlan {
    int32_t form, splits;
    int64_t partial_bytes;          // what the sums of splits need
    int32_t wide;                   // kNarrow: the side that comes from its source
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t partial_bytes_of(const ProductSize& s, int64_t splits)
{
    return splits > 1 ? splits * s.nb * ((s.na + 3) / 4 * 4) * 4 : 0;
}
// Steps of a workgroup without splits: the tiled form of 4 x 4 blocks takes all parts of B at once, against one record of A.
inline int64_t steps_of(int form, const ProductSize& s) { return form == kTiled4 || form == kNarrow ? s.groups : s.groups * s.parts; }
inline int64_t tiles_of(int form, const ProductSize& s)
{
    return (((s.na - 1) >> (5 + form)) + 1) * (((s.nb - 1) >> (5 + form)) + 1);
}

// Plans for `n` products that go in one launch where they are taken together: one form, and splits that make their
// workgroups about as long.  (What is wanted of them does not enter: the same product comes out the same bit for bit
// with and without the other.)  The time that is made least, in microseconds:
//   a workgroup's steps of a record each (direct: every wave's own) and what it takes to set up and to leave;
//   256 compute units work at once, in turns where there are more workgroups;
//   all of them together take in 16 MB a microsecond at best (a step's 68 KB of a 256 x 256 tile, fetched and not multiplied:
//   0.66 us with half of the compute units at work, 1.3 with all; multiplied, 1.05 and 1.2 to 1.5);
//   sums of splits go through memory twice, in a launch of their own.
// forced_form, forced_splits: -1 and 0, or what a tuning override asks for.
inline void product_plan(bool f4, const ProductSize* s, int n, int forced_form, int forced_splits, ProductPlan* best)
{
    // (the ends of the largest tiles: 64 K floats of a gradient, 8 x 8192 -> 16384 in 8 turns 137 us; in 4-bit products less)
    const double ends[kForms] = {0.7, 2.0, 3.2, f4 ? 12.0 : 16.0}, step[kForms] = {0.08, 0.25, 0.37, 1.15}, more_parts = 0.3;
    const double record_bytes = f4 ? 4352 : 4096;
    double best_time = 1e30;
    for (int form = 0; form < kForms; ++form) {
        if (forced_form >= 0 && form != forced_form) continue;
        int64_t tiles[2], most = 1;
        for (int i = 0; i < n; ++i) {
            tiles[i] = tiles_of(form, s[i]);
            most = steps_of(form, s[i]) > most ? steps_of(form, s[i]) : most;
        }
        for (int64_t cut = 1; cut <= kMostSplits; cut *= 2) {
            const int64_t target = ceil_div(most, cut);
            int64_t groups = 0, splits[2];
            double work = 0, longest = 0, bytes = 0, join = 0;
            for (int i = 0; i < n; ++i) {
                const int64_t all = steps_of(form, s[i]), together = form == kTiled4 ? s[i].parts : 1;
                int64_t k = forced_splits > 0 ? forced_splits : ceil_div(all, target);
                if (k > all) k = all;
                const int64_t steps = ceil_div(all, k);
                splits[i] = k = ceil_div(all, steps);               // (none of them empty)
                // (parts together: one workgroup to a compute unit, nothing to hide its ends behind)
                const double time = ends[form] + (together > 1 ? 1.2 : 0.0) + (double)steps * (step[form] + more_parts * (double)(together - 1));
                groups += tiles[i] * k;
                work += (double)(tiles[i] * k) * time;
                bytes += (double)(tiles[i] * k * steps) * (double)((1 + together) << form) * record_bytes;
                longest = time > longest ? time : longest;
                if (k > 1) join += 1.0 + 0.05 * (double)k + (double)partial_bytes_of(s[i], k) * 2 / 4e6;
            }
            // (the largest tiles one at a time, others two or more)
            double time = form == kTiled8 ? work / (double)groups * (double)ceil_div(groups, 256) : work / 256 + 0.6 * longest;
            if (time < longest || groups <= 256) time = longest;
            if (time < bytes / 16e6) time = bytes / 16e6;
            time += join > 0 ? 2.0 + join : 0.0;
            if (time < best_time) {
                best_time = time;
                for (int i = 0; i < n; ++i) best[i] = {form, (int32_t)splits[i], partial_bytes_of(s[i], splits[i]), kWideNone};
            }
            if (target == 1 || forced_splits > 0) break;
        }
    }
}

// The plan of a gradient (sizes as its job's: A is always c_in wide) with its wide side from the source, where that is worth
// a launch of its own; false: it is not.  `input`: dx = dy W, contracted over c_out; otherwise dw = dy^T x, over rows.
// From 16 M elements on of what is read once instead of written and read as operands (of each part of them): gradients of
// 7490 x 32 -> 7029 in float 110 us for 315, of 16 x 4096 -> 4096 41 for 55, of 8192 x 4096 -> 32 in bf16 48 for 61, but of 2048 x
// 64 -> 2048 in bf16 15 each for 19 both.  Weights for more than 32 rows, whose sums of splits cost more: from four times as
// many on (64 x 4096 -> 4096 in bf16 42 for 34).  More than 64 input channels: from 32 M elements on of dy's parts but the first (in
// float 4096 x 128 -> 4096 70 for 95 and 3001 x 77 -> 2999 52 for 53; in half 8192 x 100 -> 8192 202 for 268, 4096 x 128 -> 4096
// 65 for 60; in bf16 8192 x 128 -> 16384 358 for 300).
inline bool narrow_plan(const ProductSize& s, bool input, int forced_form, int forced_splits, ProductPlan* plan)
{
    if (forced_form >= 0 && forced_form != kNarrow) return false;
    const bool a_narrow = s.na <= (s.parts > 1 ? kNarrowInputs : kNarrowRows);
    if (!a_narrow && s.nb > kNarrowRows) return false;
    const int side = a_narrow ? (input ? kWideDyRows : kWideDyDown) : input ? kWideWeights : kWideInput;
    const int64_t wide = a_narrow ? s.nb : s.na, tiles = ceil_div(wide, 64);
    const int64_t worth = (int64_t)1 << (side == kWideWeights && s.nb > 32 ? 26 : 24);
    const int64_t elements = wide * s.groups * 64;
    if (forced_form < 0 && elements * (a_narrow ? s.parts : 1) < worth) return false;
    if (forced_form < 0 && a_narrow && s.na > kNarrowRows && elements * (s.parts - 1) < (int64_t)1 << 25) return false;
    // Microseconds: a step of 64 k (with three workgroups to a compute unit), their turns, and sums of splits as above.
    const double step = a_narrow ? 0.8 + 0.2 * (double)s.parts : 0.7;
    double best = 1e30;
    int64_t splits = 1;
    for (int64_t cut = 1; cut <= kMostSplits; cut += cut < 4 ? 1 : cut & (cut - 1) ? cut / 3 : cut / 2) {       // 1, 2, 3, 4, 6, 8, 12 ..
        const int64_t each = ceil_div(s.groups, forced_splits > 0 ? forced_splits : cut), k = ceil_div(s.groups, each);
        const double turns = (double)(tiles * k) / 768;
        const double time = (turns > 1 ? turns : 1) * (3.0 + step * (double)each) +
                            (k > 1 ? 3.0 + 0.1 * (double)k + (double)partial_bytes_of(s, k) * 2 / 2.5e6 : 0.0);
        if (time < best) {
            best = time;
            splits = k;
        }
    }
    *plan = {kNarrow, (int32_t)splits, partial_bytes_of(s, splits), side};
    return true;
}

}  // namespace tern
