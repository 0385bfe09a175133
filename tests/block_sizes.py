"""Sizes of which each kernel variant of the linear layers and of the norms' sums takes one: the GPU tests run them,
and tests/sanitize/host_block_plan_driver.cpp holds the library's plans to reaching every variant with them.
"""

# Rows, input width, output width. Forward, dx and dW in tiles of 256, 128 and 64, loads two or four stages ahead, one tile
# a workgroup or several, tiles shared out or not; first stages that are whole or what is left over 64; rows and columns
# that end inside tiles.
PRODUCTS = [(3257, 1880, 5328), (3257, 5328, 1880), (4699, 488, 5328), (4699, 5328, 488), (1225, 5328, 6176), (460, 2184, 11184),
            (1084, 2536, 3408), (6780, 2184, 2184), (5310, 1400, 6176), (2550, 1624, 72), (1564, 5328, 72), (2550, 72, 1624),
            (1564, 72, 5328), (6000, 1400, 1400), (1225, 3408, 9648), (17, 8312, 1024), (17, 1200, 3408), (17, 64, 64),
            (65, 568, 1024), (65, 1624, 272), (588, 1624, 72), (664, 11184, 72), (588, 72, 1624), (664, 72, 11184), (17, 664, 11184),
            (4158, 72, 72), (849, 64, 64), (1225, 488, 2536), (1225, 2536, 488), (849, 2536, 896), (849, 896, 2536),
            (2550, 768, 1024), (7662, 1200, 1624), (751, 1040, 2536), (751, 2536, 1040)]

# At most 16 rows: one, two or four pieces of K side by side in 4 or 16 waves, with K long enough that the loop over
# several runs of each wave is taken, by tiles all the same; gradients of 1, 2, 3, 4 and more rows.
FEW_ROWS = [(16, 1000, 4104), (2, 904, 16392), (1, 840, 16384), (8, 1800, 2056), (3, 1800, 8200), (3, 3464, 1032), (1, 5120, 1024),
            (12, 3272, 72), (7, 6408, 136), (2, 12680, 72), (4, 13000, 8), (5, 22008, 64), (16, 11016, 520), (6, 64, 64)]

# Batch, tokens, width, groups, tokens of a group, first token: sums over few, tens, hundreds and more parts, of few and of many
# columns, of many groups.
SUMS = [(1, 3, 264, 1, 0, 0), (1, 60, 1000, 1, 0, 0), (1, 700, 264, 1, 0, 0), (1, 600, 2056, 600, 1, 0), (2, 400, 264, 400, 1, 0),
        (1, 1100, 5120, 600, 2, 50)]
