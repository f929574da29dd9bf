"""Products of 8-bit rows and weights whose results fill whole lines, (rows, width, channels) of every variant: tile and groups of waves that share its sums, for results of 16 and of
32 bits.  Rows are ragged in all of them, channels in some."""

PITCH = 64  # results whose rows begin at multiples of this many elements fill whole lines in every type

VARIANTS = {
    (23, 768, 768): ((16, 4), (16, 4)),
    (17, 2100, 128): ((16, 8), (16, 8)),
    (500, 768, 768): ((32, 4), (32, 4)),
    (1000, 300, 1024): ((64, 1), (64, 1)),
    (3001, 1000, 960): ((64, 1), (64, 1)),
    (1000, 1040, 1024): ((64, 4), (64, 4)),
    (250, 2064, 3520): ((64, 4), (64, 4)),
    (5284, 200, 704): ((128, 1), (128, 1)),
    (3100, 144, 4032): ((128, 1), (128, 1)),
    (16380, 144, 768): ((192, 1), (192, 1)),
    (8001, 1030, 2944): ((192, 1), (192, 1)),
    (16380, 520, 2304): ((192, 1), (128, 1)),
    (4090, 300, 4096): ((256, 1), (256, 1)),
    (4001, 1040, 4032): ((256, 1), (256, 1)),
}
