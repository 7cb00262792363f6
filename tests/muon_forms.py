"""Sizes for every form of the product that takes an update's X to its next step, and which form each is meant to take.  No GPU needed."""

# which (from pairs; from the halves with another coarse step behind; from the halves with a step from pairs behind), tile, wavefronts along the sum, operands exchanged, (rows, cols)
NEXT = [
    (0, (64, 64), True, False, (257, 267)), (0, (64, 64), False, False, (1419, 1421)), (0, (128, 128), False, False, (65, 34689)), (0, (160, 256), False, False, (257, 26068)),
    (0, (160, 256), False, True, (130, 39430)), (0, (192, 256), False, False, (129, 43902)), (0, (192, 256), False, True, (194, 43899)), (0, (256, 256), False, False, (197, 49226)),
    (1, (64, 64), True, False, (257, 267)), (1, (64, 64), False, False, (257, 3309)), (1, (128, 128), False, False, (258, 11728)), (1, (160, 256), False, False, (257, 27556)),
    (1, (192, 256), False, False, (321, 27663)), (1, (192, 256), False, True, (2002, 6011)), (1, (192, 256), False, True, (6011, 2002)), (1, (192, 256), False, True, (256, 43753)),
    (1, (256, 256), False, False, (385, 24626)), (1, (192, 256), False, False, (1600, 6400)),
    (2, (64, 64), True, False, (257, 267)), (2, (64, 64), False, False, (257, 3309)), (2, (128, 128), False, False, (258, 11728)), (2, (160, 256), False, False, (257, 27556)),
    (2, (192, 256), False, False, (321, 27663)), (2, (256, 256), False, False, (256, 47803)),
]
