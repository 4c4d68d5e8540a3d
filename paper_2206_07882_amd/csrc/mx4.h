// Microscaled 4-bit floats: E2M1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), blocks of 32 neighbouring columns of
// a row with an E8M0 scale each (byte e: 2^(e-127), 255: NaN).
#pragma once

#include "qrnnt_common.h"

#define QR_MX4_BLOCK 32
#define QR_MX4_CHUNK 256   // columns of a weight tile's step: two matrix instructions of 128
#define QR_MX4_NAN 255

static inline int qr_mx4_blocks(int cols) { return (int)(((int64_t)cols + QR_MX4_BLOCK - 1) / QR_MX4_BLOCK); }
static inline int qr_mx4_pitch(int cols) { return qr_mx4_blocks(cols) * 16; }
static inline int qr_mx4_scale_pitch(int cols) { return qr_round_up(qr_mx4_blocks(cols), 8); }
static inline int qr_mx4_chunks(int cols) { return qr_mx4_scale_pitch(cols) / 8; }

// Packed weights: first the codes, for every [row tile of 16][chunk] two blocks of 1 KiB, each the operand of one matrix
// instruction as it is: lane l's 16 bytes at 16*l of block h are block 8*chunk + 2*(l/16) + h of row 16*tile + l%16.  (A lane of
// group g takes the blocks 2g and 2g + 1 in the two instructions, so that its two scales lie side by side; the activations
// are read in the same order.)  Then the scales, 128 bytes for every [row tile][chunk]: the chunk's 8 scales of 16 rows.
static inline size_t qr_mx4_tiles(int rows, int cols) { return (size_t)((rows + 15) / 16) * qr_mx4_chunks(cols); }
static inline size_t qr_mx4_packed_bytes(int rows, int cols) { return qr_mx4_tiles(rows, cols) * (2048 + 128); }
