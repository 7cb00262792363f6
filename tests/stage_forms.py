"""Sizes for every form that the calls of a stage's training step have, and which form each is meant to take.  numpy and torch only; no GPU needed."""
import torch

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32

# type, sides of a tile, each load bounded for itself, tokens shared out, (rows, n_out, n_in): odd sizes, tokens that end inside a tile of them, and last
# tiles that begin inside the ones before them
WEIGHT_GRADIENTS = [
    (BF16, (64, 64), True, False, (209, 37, 34)), (BF16, (64, 64), True, True, (731, 35, 36)),
    (BF16, (64, 64), False, False, (200, 71, 69)), (BF16, (64, 64), False, True, (938, 71, 72)),
    (BF16, (128, 128), False, False, (206, 193, 11320)), (BF16, (128, 128), False, True, (2645, 5105, 194)),
    (BF16, (256, 128), False, False, (759, 19819, 152)), (BF16, (256, 128), False, True, (5106, 4607, 140)),
    (BF16, (256, 192), False, False, (398, 21743, 513)), (BF16, (256, 192), False, True, (5971, 7997, 271)),
    (BF16, (256, 256), False, False, (357, 32331, 469)), (BF16, (256, 256), False, True, (5313, 393, 9990)),
    (F16, (64, 64), True, False, (206, 43, 33)), (F16, (64, 64), True, True, (397, 35, 35)),
    (F16, (64, 64), False, False, (206, 75, 71)), (F16, (64, 64), False, True, (568, 75, 70)),
    (F16, (128, 128), False, False, (202, 135, 15032)), (F16, (128, 128), False, True, (5023, 197, 1230)),
    (F16, (256, 128), False, False, (3352, 31047, 138)), (F16, (256, 128), False, True, (53806, 1727, 150)),
    (F16, (256, 256), False, False, (201, 21091, 656)), (F16, (256, 256), False, True, (2768, 7125, 385)),
    (F32, (64, 64), True, False, (202, 33, 35)), (F32, (64, 64), True, True, (341, 35, 37)),
    (F32, (64, 64), False, False, (206, 75, 71)), (F32, (64, 64), False, True, (391, 71, 69)),
    (F32, (128, 128), False, False, (206, 5707, 134)), (F32, (128, 128), False, True, (1004, 133, 1933)),
    (F32, (256, 128), False, False, (209, 16755, 135)), (F32, (256, 128), False, True, (1170, 5487, 143)),
    (F32, (256, 256), False, False, (214, 22933, 273)), (F32, (256, 256), False, True, (1827, 267, 5509)),
]
# sizes as models have them, multiples of 64: the first projection behind a layer norm of 1600 features, and others
MODEL_SIZES = [(BF16, (256, 192), (4096, 6400, 1600)), (BF16, (128, 128), (512, 1024, 4096)), (F16, (256, 256), (1024, 4096, 4096)), (F32, (256, 256), (320, 4096, 4096))]

# lanes to a row, octets of a row to a lane, (rows, cols): more rows than are under way at a time, so that teams go round, some of them one time less
BACKWARD = [(8, 1, (40001, 40)), (16, 1, (20003, 100)), (32, 1, (9001, 250)), (64, 1, (5003, 511)), (64, 2, (5000, 768)), (64, 2, (2101, 1023)), (256, 1, (2101, 1601)),
            (256, 1, (3000, 1600)), (256, 2, (1303, 4095)), (512, 2, (1101, 8190)), (512, 4, (600, 16379))]
FORWARD = [(8, 1, (70001, 40)), (16, 1, (40001, 100)), (32, 1, (20001, 250)), (64, 1, (9001, 511)), (64, 2, (5001, 1023)), (128, 2, (2501, 1601)), (128, 2, (2500, 1600)),
           (256, 2, (1301, 4095)), (512, 2, (701, 8190)), (512, 4, (601, 16379)), (1024, 4, (603, 32767))]
