// maps.cuh -- tensor maps of the layer operators (defined in linear.cu).
#pragma once

namespace rdn {
// bf16 [depth][rows][cols] whose rows are ld elements apart (rows * ld from one index of the first axis to
// the next), boxes of box_cols x box_rows, no swizzle; out of range reads as zero and is not written.
// false if the driver's encoder is unavailable or refuses.
bool make_rows_map(void *map128, const void *p, int cols, int rows, int depth, long long ld, int box_cols,
                   int box_rows);
}  // namespace rdn
