// What the kernels that orthogonalise matrices are told about them (by value).
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace cb {

constexpr int kOrthoTable = 40;

struct OrthoMatrix {
    const void* in;
    void* out;
    size_t x, y, a, b;                               // places in the workspace: X of even and of odd steps, A, B
    int m, n, mp, np;                                // m <= n, and both rounded up to whole tiles
    uint32_t chunk0, side0, square0, apply0;         // its first workgroups, and tiles
    uint8_t bf16, tall;                              // tall: in and out are n x m
};
// Workgroups are dealt to the eight XCDs in turn: tiles from one end to the next are one XCD's, one after the other.
constexpr int kXcds = 8;
struct OrthoEnds { uint32_t of[kXcds + 1]; };
struct OrthoTable {
    OrthoMatrix of[kOrthoTable];
    OrthoEnds gram, square, apply;
    int n;
};
static_assert(sizeof(OrthoTable) <= 3800, "kernel arguments");

}  // namespace cb
