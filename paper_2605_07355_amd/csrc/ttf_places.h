// Index arithmetic of the attention kernels that decides what they read: plain constant expressions, the same on the host.
#pragma once

namespace ttf {

// Lane group g (of four) takes the 16-byte pieces 4 s + g of a head of head_dim entries of entry_bytes.  Whether the head has that piece.
constexpr bool has_piece(int s, int g, int head_dim, int entry_bytes) { return (s * 64 + g * 16) / entry_bytes < head_dim; }
// Where the group's first piece is.  A group that the head has nothing for stands at its start (and takes 0 for what it reads there).
constexpr int first_piece(int g, int head_dim, int entry_bytes) { return has_piece(0, g, head_dim, entry_bytes) ? 16 * g : 0; }
// How far from there its s-th is; where the head has none, the first again.
constexpr int next_piece(int s, int g, int head_dim, int entry_bytes) { return has_piece(s, g, head_dim, entry_bytes) ? s * 64 : 0; }

// Whether the lane-th page from `page` on, of page_size slots, begins before entry `stop`.  (Pages of one slot and a window over entries near 2^31:
// the number is past 31 bits.)
constexpr bool page_begins(int page, int lane, int page_size, int stop) { return (long long)((unsigned)page + (unsigned)lane) * page_size < stop; }

}  // namespace ttf
