// Attention over pages of 8-bit rows with a scale for each row and head: with codes K'[j], V'[j] and scales ks[j], vs[j],
//   z_j = scale ks[j] (q[b][h] . K'[j]),   o[b][h] = sum_j w_j V'[j] / sum_j p_j,   p_j = exp(z_j - max),   w_j = p_j vs[j].
// The kernel is that of the wider types (attention_paged.h): a unit of V is 16 rows of a dim, a lane's 16 bytes of K are 16 dims, and a turn of 16 loads a lane holds twice the rows.
//  * Codes go into the products as fp16, which holds every code of both types: e4m3 by the conversion instruction, two at a time; whole numbers by putting the bytes into the last digits of 1024 ... 1279 and subtracting
//    1152, five instructions for four.  q and w are two fp16 halves, as over fp16 rows: products and sums lose nothing to the 8 bits.
//  * A lane loads the scales of one row of each group; the 16 lanes side by side have those of the 16 rows that each of them has scores of, so a factor per row is an operand of the multiplication itself (the
//    lane's neighbour by DPP), one instruction a score and one a weight.
//  * Scales have 32 bits and weights times scales any size, but fp16 halves need them below 2^16 and not far below: every head keeps a power of two above its largest w so far (unit, a whole exponent: what goes from one unit to
//    the next is exact), brings that w to 32752 at least and 65504 at most, fp16's largest, and rescales its sums when it grows, apart from the maximum of the scores, which the sum of the p_j goes by.  A row with a large value and no weight does not cost the others digits.
//
// Bound by memory where there is much of it: 32 x 2304 rows of 32 heads, e4m3, 107 us = 5.9 TB/s (fp16 rows 189 to 195 us, 6.3), i8 108.5; 48 requests of 1 to 32768 rows of 8 heads, i8, 66 us = 5.1 TB/s (109 and 6.0).  What is
// left is as long as over fp16 rows (12 to 15 us: ramp, a first turn of every (sequence, heads) with nothing beside it, joins) and weighs twice as much.  Small launches are 0.5 to 1 us longer than over fp16 rows (640 rows of 32 heads 9.3 to 9.6 us, 8.9): a
// turn has twice the rows.  us before and after: scratch for 10 to 25 registers, in the beginnings of (sequence, heads) alone, against none, i8 32 x 2304 119.8 / 108.9, ragged 77.2 / 65.7, 640 rows 10.8 / 9.8 (hence the lane's number and the
// reciprocals computed in the loop); masks from constants that are kept against the number of rows left 118 / 107.8, ragged 77.7 / 65.8; the next turn's K requested ahead of the scores into registers of its own
// 107 / 108, ragged 65.6 / 73.4 (not kept); conversions placed between the products of the group before: no difference (not kept); sums
// brought to a new maximum in a branch of their own 12.62, beside the exponentials 12.50, and the scale taken apart by the host 12.40 (8 x 1152 rows of 8 heads, 8 query heads each).
#include "attention_paged.h"

namespace d3 {

int launch_attention_paged8(const PagedAttnArgs& a, int hd, int kv_dtype, int n_cu, hipStream_t s) {
    if (kv_dtype == D3_I8) return hd == 64 ? launch<i8_t, 64>(a, n_cu, s) : launch<i8_t, 128>(a, n_cu, s);
    if (kv_dtype == D3_E4M3) return hd == 64 ? launch<e4m3_t, 64>(a, n_cu, s) : launch<e4m3_t, 128>(a, n_cu, s);
    return (int)hipErrorInvalidValue;
}

}  // namespace d3
