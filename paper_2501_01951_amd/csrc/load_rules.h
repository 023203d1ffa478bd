// Which addresses of a row are read where a lane takes more than one 16-byte group.  Plain C++, so that the host can check it.
#pragma once

namespace mixgcn {

// A lane takes the fp32 columns col .. col + 7 of a row of `cols` (col a multiple of 4, below cols) as two groups of four; the
// first column of the second group, or col again where that group has no column of the matrix.  A matrix may be some columns
// of a wider one: its rows' pitch does not say what lies behind its columns, and behind those of its last row nothing may.
constexpr int second_group(int col, int cols) { return col + 4 < cols ? col + 4 : col; }

}  // namespace mixgcn
