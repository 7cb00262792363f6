"""Sizes for every form that products in 8-bit floating point and updates of weights have, and which form each is meant to take.  No GPU needed."""
import torch

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32

# type, (side of a tile or 0 for a few tokens, wavefronts along the sum, sum shared out, last tiles in quarters), (rows, n_out, n_in): odd sizes, tiles that end outside the matrix
PRODUCTS = [
    (BF16, (0, False, False, False), (7, 33, 391)), (BF16, (0, False, False, False), (31, 257, 1155)),
    (BF16, (64, True, False, False), (45, 77, 903)), (BF16, (64, True, True, False), (35, 70, 5256)),
    (BF16, (64, False, False, False), (1027, 2051, 515)), (BF16, (64, False, True, False), (4210, 7, 11138)),
    (BF16, (128, False, False, False), (1500, 5003, 389)), (BF16, (128, False, True, False), (11242, 77, 7172)),
    (BF16, (256, False, False, False), (3001, 4099, 900)), (BF16, (256, False, False, True), (16100, 6300, 390)), (BF16, (256, False, True, False), (134, 5741, 58402)),
    (F32, (0, False, False, False), (7, 33, 391)), (F32, (64, True, False, False), (45, 77, 903)), (F32, (64, True, True, False), (35, 70, 5256)),
    (F32, (64, False, False, False), (1027, 2051, 515)), (F32, (64, False, True, False), (16946, 5, 2491)),
    (F32, (128, False, False, False), (1500, 5003, 389)), (F32, (128, False, True, False), (11113, 81, 10687)),
    (F32, (256, False, False, False), (3001, 4099, 900)), (F32, (256, False, False, True), (16100, 6300, 390)), (F32, (256, False, True, False), (10475, 491, 15257)),
]

# which of an update's eight products, its tile, wavefronts along the sum, sum shared out, (rows, cols)
UPDATES = [
    (0, (64, 64), True, False, (257, 300)), (0, (64, 64), True, True, (70, 3001)), (0, (64, 64), False, False, (1927, 1983)), (0, (64, 64), False, True, (1419, 1421)),
    (0, (128, 128), False, False, (3221, 3306)), (0, (128, 128), False, True, (1765, 1781)), (0, (256, 256), False, False, (4938, 4891)), (0, (256, 256), False, True, (3745, 1947)),
    (1, (64, 64), True, False, (257, 300)), (1, (64, 64), False, False, (1927, 1983)), (1, (64, 64), False, True, (1419, 1421)), (1, (128, 128), False, False, (3221, 3306)),
    (1, (128, 128), False, True, (1765, 1781)), (1, (256, 256), False, False, (4938, 4891)), (1, (256, 256), False, True, (2978, 2993)),
    (2, (64, 64), True, False, (257, 300)), (2, (64, 64), False, False, (1419, 1421)), (2, (128, 128), False, False, (65, 36734)), (2, (160, 256), False, False, (129, 39956)),
    (2, (192, 256), False, False, (161, 43484)), (2, (256, 256), False, False, (193, 49487)),
    (3, (64, 64), True, False, (257, 300)), (3, (64, 64), False, False, (1419, 1421)), (3, (128, 128), False, False, (65, 36734)), (3, (160, 256), False, False, (129, 39956)),
    (3, (192, 256), False, False, (129, 43515)), (3, (256, 256), False, False, (130, 49756)),
    (4, (64, 64), True, False, (257, 267)), (4, (64, 64), True, True, (1805, 259)), (4, (64, 64), False, True, (1419, 1421)), (4, (128, 128), False, False, (3090, 3110)),
    (4, (128, 128), False, True, (1483, 1555)), (4, (256, 256), False, False, (4529, 4554)), (4, (256, 256), False, True, (1937, 4890)),
    (5, (64, 64), True, False, (257, 267)), (5, (64, 64), False, True, (1419, 1421)), (5, (128, 128), False, False, (3090, 3110)), (5, (128, 128), False, True, (1683, 1697)),
    (5, (256, 256), False, False, (4529, 4554)), (5, (256, 256), False, True, (2889, 2839)),
    (6, (64, 64), True, False, (257, 267)), (6, (64, 64), False, False, (3322, 257)), (6, (128, 128), False, False, (11972, 258)), (6, (160, 256), False, False, (259, 27609)),
    (6, (192, 256), False, False, (27991, 324)), (6, (256, 256), False, False, (25357, 386)),
    (7, (64, 64), True, False, (257, 267)), (7, (64, 64), False, False, (3322, 257)), (7, (128, 128), False, False, (11972, 258)), (7, (160, 256), False, False, (27578, 263)),
    (7, (192, 256), False, False, (27991, 324)), (7, (256, 256), False, False, (257, 31178)),
]
