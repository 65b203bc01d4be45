// Rows of a sequence from the starts of packed sequences, whatever these hold.  Plain C++ without a HIP header, so that a host program can go over them
// (tests/host/starts_check.cpp).
#pragma once

namespace lss {

// A start within a tensor of `rows` rows
constexpr int start_within(int start, int rows) { return start < 0 ? 0 : start < rows ? start : rows; }
// Rows from one start to the next: 0 .. rows.  (Both are brought into range first: a next one of -2^31 less a begin above 0 would be 2^31 - .. in 32 bits.)
constexpr int rows_between(int start, int next, int rows)
{
    const int n = start_within(next, rows) - start_within(start, rows);
    return n < 0 ? 0 : n;
}

} // namespace lss
