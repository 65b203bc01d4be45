// The workgroup's form of a packed bf16 forward launch, from what the host knows: rows, keys and sequences, not the sequences' lengths.  Plain C++
// without a HIP header, so that a host program can go over the choices.
#pragma once
#include <stdint.h>

namespace lss {

// Blocks of 32 rows x groups of wavefronts that have a part of the keys each
struct PackedForm { int row_blocks, groups; };

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
inline PackedForm pick_packed_form(int64_t rows_q, int64_t rows_k, int64_t B, int64_t H, int64_t H_kv, int64_t d)
{
    const double rows = (double)rows_q * (double)(H / H_kv) / (double)B, keys = (double)rows_k / (double)B;
    const double tiles = rows / 128.0 + 0.5, W = (double)(B * H_kv) * (tiles > 1.0 ? tiles : 1.0);
    if (d == 64) {
        if (W > 512.0 || (W > 256.0 && keys < 4096.0)) return {4, 1};
        if (W > 256.0) return {4, 2};
        if (keys < 160.0) return {2, 1};
        if (W <= 64.0) return {1, 4};
        return W <= 144.0 && keys >= 2048.0 ? PackedForm{2, 4} : PackedForm{2, 2};
    }
    if (W > 512.0) return W >= 1024.0 && keys >= 4096.0 ? PackedForm{8, 1} : PackedForm{4, 1};
    if (W > 256.0) return keys >= 4096.0 ? PackedForm{4, 2} : PackedForm{4, 1};
    if (keys < 64.0 || (W > 144.0 && keys < 1024.0)) return {4, 1};
    return {2, 2};
}

} // namespace lss
