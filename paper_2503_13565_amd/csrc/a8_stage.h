// Where the direct loads of the 8-bit product's blocks (gemm_a8.hip, gemm_a8_mid.hip) read: a phase of steps of 128 along K, of rows that lie
// one behind the other, in pieces of 16 bytes.  Plain integer arithmetic without any device header, so that every lane's load can be walked on the CPU.
//
// A load's address is the descriptor's base plus a lane offset plus a scalar offset, and it is in range where the lane offset is below the
// descriptor's bytes less the scalar offset.  That difference is unsigned: so the scalar offset stays within the descriptor whatever is asked for, and what
// is not there (rows behind the last, pieces behind K) has a lane offset beyond any descriptor.
#pragma once

namespace mxfp4 {
namespace a8 {

constexpr int kOob = 0x7FFFFFF0;        // lane offset beyond any descriptor: the load returns zero

// 0 where at <= last, else an offset beyond any descriptor (arithmetic, as a branch around a load makes the compiler wait for it).
constexpr int past(int last, int at) { return ((last - at) >> 31) & kOob; }

// Which of a row's chunks of 16 bytes (a power of two) takes the first place: 256 bytes of the LDS then hold sixteen rows' chunks of
// one number, so that the sixteen lanes that a turn of the LDS serves find sixteen different places.
constexpr int turn(int row, int chunks) { return chunks >= 16 ? row & 15 : row / (16 / chunks) & (chunks - 1); }

// Piece `piece` of a block's phase of `chunks` pieces a row: its row, its chunk, and where that lies behind the first row's first piece of the phase.
constexpr int piece_row(int piece, int chunks) { return piece / chunks; }
constexpr int piece_chunk(int piece, int chunks) { return piece % chunks ^ turn(piece_row(piece, chunks), chunks); }
constexpr int piece_offset(int piece, int chunks, int rows, int row_bytes)
{
    return (piece_row(piece, chunks) * row_bytes + piece_chunk(piece, chunks) * 16) | past(rows - 1, piece_row(piece, chunks));
}

// The phase from step `step` on, of `steps`; a step is `step_bytes` of a row.  The scalar offset (of a phase behind the last: the last step's, as `steps`
// steps may be more than a descriptor of a row or two has), and the first chunk of the row.
constexpr int phase_from(int step, int steps, int step_bytes) { return (step < steps ? step : steps - 1) * step_bytes; }
constexpr int phase_chunk(int step, int step_bytes) { return step * (step_bytes / 16); }

}  // namespace a8
}  // namespace mxfp4
