// Layout of a layer packed to 4 bits, shared by the kernels that write and read it.
//
// Codes lie in tiles of 16 rows x 128 columns, 1 KB each, tile (rb, kt) at index rb * KT + kt.  Lane
// l = 16 quad + n of a wavefront owns 16 bytes of a tile: row n, and in its dword s the eight columns
// 32 s + 8 quad + 0..7.  So dword s of all lanes is one operand of a 16x16x32 matrix instruction whose 32
// columns are consecutive (a group of 32 ends between two instructions), and a wavefront reads a tile with
// one contiguous 16-byte load per lane.  Within a dword nibble i holds column 2 i and nibble i + 4 column
// 2 i + 1: shifting the dword puts the pair (2 i, 2 i + 1) in the same place of both its halves, so one shift
// and one and-or turn two codes into two 16-bit numbers.
//
// Steps and offsets follow the codes, two half-precision numbers in 4 bytes.  Groups of 128 columns and
// more: entry (rb, g, n) at (rb * NG + g) * 16 + n.  Groups of 32 or 64: the SUB = 128 / group entries of a tile's
// row together, (rb, kt, n, sub) at ((rb * KT + kt) * 16 + n) * SUB + sub, one load per lane and tile.
// What pads the last tiles has code, step and offset 0.
#pragma once

#include "common.h"

struct pack4_layout {
    int R, d, RB, KT;
    int SUB;          // groups of a tile (1, 2 or 4)
    int tpg;          // tiles of a group (1 where SUB > 1)
    int NG;           // groups of a row as the caller counts them, ceil(d / group)
    size_t scales;    // byte offset of the steps
    size_t bytes;
};

// false: not a group size the packed form has
static inline bool pack4_layout_of(int R, int d, int group, pack4_layout *L)
{
    if (group < 0 || (group > 0 && group < d && group != 32 && group != 64 && group % 128 != 0)) return false;
    L->R = R;
    L->d = d;
    L->RB = R / 16 + (R % 16 != 0);
    L->KT = d / 128 + (d % 128 != 0);
    const bool one = group == 0 || group >= d;
    L->SUB = one || group >= 128 ? 1 : 128 / group;
    L->tpg = one ? L->KT : group >= 128 ? group / 128 : 1;
    L->NG = one ? 1 : (int)(((int64_t)d + group - 1) / group);
    L->scales = (size_t)L->RB * L->KT * 1024;
    const size_t entries = L->SUB > 1 ? (size_t)L->RB * L->KT * 16 * L->SUB : (size_t)L->RB * L->NG * 16;
    L->bytes = L->scales + 4 * entries;
    return true;
}
