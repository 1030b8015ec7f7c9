"""Sizes of 4-bit products for every kernel that there is, with the one that each takes
and the parts of its sum, on 256 compute units: (form and parts for fp32 results, the
same for 16-bit ones).  Used on the CPU, which asks for the choice, and on the GPU,
which asks again and runs it."""

# rows, columns, results
PRODUCTS = {
    "large": ((3500, 3000, 3501), ("tile_256", 1), ("tile_256", 1)),
    "large_odd_stages": ((3401, 3328, 3588), ("tile_256", 1), ("tile_256", 1)),
    "large_16_bit": ((3500, 2048, 3501), ("tile_128_short", 1), ("tile_256", 1)),
    "large_16_bit_odd_stages": ((3473, 2300, 3555), ("tile_128_short", 1), ("tile_256", 1)),
    "tiles_short_sum": ((2001, 300, 1999), ("tile_128_short", 1), ("tile_128_short", 1)),
    "tiles_narrow": ((20003, 100, 301), ("tile_128_short", 1), ("tile_128_short", 1)),
    "tiles": ((1500, 1400, 1501), ("tile_128", 1), ("tile_128", 1)),
    "tiles_odd_stages": ((1501, 1500, 1500), ("tile_128", 1), ("tile_128", 1)),
    "tiles_deep_1": ((1401, 256 * 24 + 1, 1476), ("tile_128_deep", 1), ("tile_128_deep", 1)),
    "tiles_deep_2": ((1400, 256 * 26, 1477), ("tile_128_deep", 1), ("tile_128_deep", 1)),
    "tiles_deep_3": ((1399, 256 * 26 + 100, 1475), ("tile_128_deep", 1), ("tile_128_deep", 1)),
    "tiles_deep_4": ((1398, 256 * 28 - 3, 1474), ("tile_128_deep", 1), ("tile_128_deep", 1)),
    "parts_wide": ((701, 256 * 48 - 5, 699), ("tile_128_deep", 3), ("tile_128_deep", 3)),
    "parts_wide_last": ((700, 256 * 63, 702), ("tile_128_deep", 4), ("tile_128_deep", 4)),
    "parts_wide_few": ((770, 256 * 34, 771), ("tile_128_deep", 2), ("tile_128_deep", 2)),
    "parts": ((260, 256 * 80 - 5, 303), ("tile_128_deep", 12), ("tile_128_deep", 12)),
    "parts_small": ((70, 256 * 70, 71), ("tile_128_deep", 14), ("tile_128_deep", 14)),
    "parts_one_row": ((1, 256 * 70, 41), ("tile_128_deep", 14), ("tile_128_deep", 14)),
    "parts_sixteen": ((5, 256 * 64, 43), ("tile_128_deep", 16), ("tile_128_deep", 16)),
    "parts_many": ((130, 256 * 260 + 9, 67), ("tile_128_deep", 53), ("tile_128_deep", 53)),
    "thirty_two": ((300, 2048, 1001), ("rows_32", 1), ("rows_32", 1)),
    "thirty_two_odd": ((401, 1500, 999), ("rows_32", 1), ("rows_32", 1)),
    "thirty_two_long": ((500, 256 * 40, 501), ("rows_32", 1), ("rows_32", 1)),
    "sixteen": ((9, 3001, 333), ("rows_16", 1), ("rows_16", 1)),
    "sixteen_no_parts_yet": ((260, 256 * 40 - 5, 300), ("rows_16", 1), ("rows_16", 1)),
    "sixteen_four_waves": ((33, 2600, 3001), ("rows_16_short", 1), ("rows_16_short", 1)),
    "sixteen_short": ((17, 1000, 19), ("rows_16_short", 1), ("rows_16_short", 1)),
    "along": ((3001, 100, 303), ("rows_16_along", 1), ("rows_16_along", 1)),
    "along_few_rows": ((16, 131, 20001), ("rows_16_along", 1), ("rows_16_along", 1)),
    "along_narrow": ((16449, 33, 5), ("rows_16_along", 1), ("rows_16_along", 1)),
    "along_square": ((1003, 250, 999), ("rows_16_along", 1), ("rows_16_along", 1)),
}

# rows, experts of each, experts, columns, results
EXPERTS = {
    "large": ((2941, 2, 2, 256 * 40 - 180, 5881), ("tile_256", 1), ("tile_256", 1)),
    "large_odd_stages": ((5889, 1, 1, 256 * 41, 5870), ("tile_256", 1), ("tile_256", 1)),
    "tiles_short_sum": ((2501, 2, 7, 300, 301), ("tile_128_short", 1), ("tile_128_short", 1)),
    "tiles_many": ((1793, 2, 3, 2060, 3001), ("tile_128_short", 1), ("tile_128_short", 1)),
    "tiles": ((501, 2, 5, 2000, 1501), ("tile_128", 1), ("tile_128", 1)),
    "tiles_few_of_each": ((31, 2, 11, 256 * 17 + 3, 5538), ("tile_128", 1), ("tile_128", 1)),
    "tiles_deep": ((1001, 2, 4, 6200, 701), ("tile_128_deep", 1), ("tile_128_deep", 1)),
    "tiles_deep_odd": ((500, 1, 4, 256 * 24 + 1, 700), ("tile_128_deep", 1), ("tile_128_deep", 1)),
    "thirty_two": ((300, 1, 2, 1100, 1301), ("rows_32", 1), ("rows_32", 1)),
    "thirty_two_eight": ((267, 3, 8, 1000, 300), ("rows_32", 1), ("rows_32", 1)),
    "thirty_two_sixteen": ((1025, 2, 16, 512, 129), ("rows_32", 1), ("rows_32", 1)),
    "sixteen": ((300, 1, 2, 1100, 131), ("rows_16", 1), ("rows_16", 1)),
    "sixteen_four_waves": ((550, 2, 5, 900, 140), ("rows_16_short", 1), ("rows_16_short", 1)),
    "along": ((41, 3, 60, 1030, 1111), ("rows_16_along", 1), ("rows_16_along", 1)),
    "along_eight_of_each": ((200, 2, 50, 40, 2079), ("rows_16_along", 1), ("rows_16_along", 1)),
}


def chosen(case, dtype):
    """The form and parts that `case` names for results of a type."""
    return case[1] if dtype == "f32" else case[2]
