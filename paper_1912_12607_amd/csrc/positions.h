// Rotary positions and page tables: argument structs, launchers (token_positions.hip).
#pragma once
#include "tokens.h"

namespace int8t {

struct RotateTensor {
    const void* x;
    void* y;                 // may be x
    size_t x_token, x_head, y_token, y_head;      // pitches, elements
    int heads;
    int wide_x, wide_y;      // 16-byte accesses of the heads' first values
};
struct RotateArgs {
    RotateTensor t[2];       // the second one's heads may be 0
    const int* positions;
    const double* turns;     // rot / 2: of a pair per position, in whole turns
    int tokens, dim, rot, type;
    int interleaved, back;   // pairs (2 i, 2 i + 1) instead of (i, i + rot / 2); by the negative angle
    float amplitude;
};
hipError_t launch_rotate(const RotateArgs& a, hipStream_t st);

struct PagesArgs {
    const int *have, *add;   // tokens of the requests, new ones; shrink: those that stay
    int* table;
    size_t table_pitch;
    const int* free;         // shrink: written
    const int* available;
    int requests, width, page_size, pages, tokens;
    FastDiv by_page;
    int *lengths, *left, *starts, *positions, *without;      // out; left: available pages
    long long* slots;
};
hipError_t launch_pages_extend(const PagesArgs& a, hipStream_t st);
hipError_t launch_pages_shrink(const PagesArgs& a, hipStream_t st);

}  // namespace int8t
