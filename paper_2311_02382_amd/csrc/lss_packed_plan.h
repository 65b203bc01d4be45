// The workgroups' form of a packed forward launch and its key splits, from what the host knows: rows, keys and sequences, not the sequences' lengths.  Plain C++
// without a HIP header, so that a host program can go over the choices.
#pragma once
#include <stdint.h>

namespace lss {

// Blocks of 32 rows x groups of wavefronts that have a part of the keys each; key splits
struct PackedPlan { int row_blocks, groups, splits; };

// W: workgroups of 128 rows that the sequences would make if they were about as long as each other; keys: of an average sequence.  108 launches in every
// form (1 to 30 sequences of 1 to 8192 rows behind 0 to 8000 keys, 8 to 32 heads with 1 to 32 of keys, both head widths), us:
//   * W > 512, all compute units have several: 4 x 1, three to a compute unit at d = 64 and two at d = 128.  Eight sequences of 750 to
//     2250 rows, 32 heads, 8 of keys: d = 64 124 (2 x 2: 171), d = 128 209 (8 x 1: 227, 4 x 2: 286).  Long sequences at d = 128: 8 x 1, 256 rows that share a
//     tile: 16 heads of 8192 rows 256 (4 x 1: 271).
//   * Up to two workgroups a compute unit, long walks: two groups, 4 x 2: 8 heads of 8192 rows d = 64 89 (4 x 1: 100), d = 128 148 (170); 32 of 2048 rows,
//     where 4 x 1 is as good: 33 (30) and 51 (50).
//   * Up to one: smaller workgroups.  8 heads of 4096 rows: 2 x 2 33 (4 x 1: 50) and 58 (74).  A quarter of the compute units, d = 64: four groups of 32 rows,
//     8 heads of 1024 rows 10.4 (2 x 2: 12.2); up to half of them and long walks 2 x 4, 8 heads of 512 rows behind 8000 51 (57).
//   * Short sequences have nothing to divide: 16 sequences of 100 rows, 8 heads: d = 64 2 x 1 7.3 (2 x 2: 7.9), d = 128 from two a
//     compute unit on 4 x 1: 16 of 16 heads 10.9 (2 x 2: 17.1).
inline PackedPlan pick_packed_form(double W, double keys, int64_t d)
{
    if (d == 64) {
        if (W > 512.0 || (W > 256.0 && keys < 4096.0)) return {4, 1, 1};
        if (W > 256.0) return {4, 2, 1};
        if (keys < 160.0) return {2, 1, 1};
        if (W <= 64.0) return {1, 4, 1};
        return W <= 144.0 && keys >= 2048.0 ? PackedPlan{2, 4, 1} : PackedPlan{2, 2, 1};
    }
    if (W > 512.0) return W >= 1024.0 && keys >= 4096.0 ? PackedPlan{8, 1, 1} : PackedPlan{4, 1, 1};
    if (W > 256.0) return keys >= 4096.0 ? PackedPlan{4, 2, 1} : PackedPlan{4, 1, 1};
    if (keys < 64.0 || (W > 144.0 && keys < 1024.0)) return {4, 1, 1};
    return {2, 2, 1};
}
// Key splits, whose results a second launch joins (3 to 4 us): where few workgroups walk many keys.
//   * bf16, up to 40 workgroups of 128 rows (64 at d = 128), 2048 keys: 2 x 2, up to 256 workgroups and eight splits.  64 rows behind 4000 keys, 32 heads, 8 of
//     keys: d = 64 21.8 -> 15, d = 128 47.2 -> 20; 300 behind 30,000, 8 heads, 2 of keys: 124 -> 42, 301 -> 67.  From 64 workgroups on nothing is gained, four
//     groups in a workgroup do as well (8 x 8 heads of 16 rows behind 1000: 10.3, 2 splits 12.6).
//   * float has no groups: as many as the chip holds at once, 128 keys each at least.  8 heads of 2048 rows: d = 64 104 -> 52, d = 128 180 -> 78; of 4096 rows,
//     with three: 204 -> 122, 369 -> 200; 16 sequences of a row behind 3000 keys at d = 128 280 -> 96 with four (six: 123).
inline PackedPlan pick_packed_plan(int64_t rows_q, int64_t rows_k, int64_t B, int64_t H, int64_t H_kv, int64_t d, int elem_bytes)
{
    const double rows = (double)rows_q * (double)(H / H_kv) / (double)B, keys = (double)rows_k / (double)B;
    const double tiles = rows / 128.0 + 0.5, W = (double)(B * H_kv) * (tiles > 1.0 ? tiles : 1.0);
    const auto up_to = [](double x, double most) { return x < 1.0 ? 1 : (int)(x < most ? x : most); };
    if (elem_bytes == 4) {
        const int fill = up_to((d == 64 || W > 200.0 ? 768.0 : 560.0) / W, 16.0);
        return {4, 1, up_to(keys / 128.0, fill)};
    }
    if (W <= (d == 64 ? 40.0 : 64.0) && keys >= 2048.0) return {2, 2, up_to(128.0 / W, 8.0)};
    return pick_packed_form(W, keys, d);
}

} // namespace lss
