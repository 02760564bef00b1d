"""Sizes of forward calls in 8 bits for each kernel with an epilogue of its own: (pair, M, K, N) and the kernel that the rules of csrc/q8_plan.h
choose there; whole tiles and tiles that end outside the results."""

SIZES = {
    (0, 256, 129, 256): "fwd 64x64", (0, 73, 138, 8525): "fwd 64x64 many", (0, 36, 2923, 32): "fwd 64x64 divided",
    (0, 133, 131, 11251): "fwd 128x128", (0, 1280, 136, 3328): "fwd 128x128 many",
    (0, 1280, 2453, 3328): "fwd 256x128", (0, 2497, 2479, 1605): "fwd 256x128", (0, 5518, 2181, 3843): "fwd 256x128 many",
    (0, 7168, 259, 1792): "fwd 256x256", (0, 2854, 260, 4286): "fwd 256x256", (0, 6585, 8644, 547): "fwd 256x256 divided",
    (0, 7168, 135, 3584): "fwd 256x256 many", (0, 3516, 131, 6966): "fwd 256x256 many",
    (1, 256, 129, 256): "fwd pair 64x128", (1, 66, 143, 8576): "fwd pair 64x128 many", (1, 37, 923, 35): "fwd pair 64x128 divided",
    (1, 69, 296, 8256): "fwd pair 128x128", (1, 2560, 136, 1280): "fwd pair 128x128 many", (1, 4182, 1459, 68): "fwd pair 128x128 divided",
    (1, 256, 2453, 8448): "fwd pair 256x128", (1, 139, 3091, 10927): "fwd pair 256x128", (1, 2482, 3666, 3223): "fwd pair 256x128 many",
    (1, 1024, 129, 4096): "fwd pair 256x256", (1, 431, 130, 8299): "fwd pair 256x256", (1, 2816, 5213, 768): "fwd pair 256x256 divided",
    (1, 768, 130, 11008): "fwd pair 256x256 many", (1, 5037, 132, 1580): "fwd pair 256x256 many",
}
