"""Sizes that lead a linear layer through each of its kernels, and where the library's
rules lead them: test_block_host.py holds the rules to it on the CPU, so that the GPU
tests that run these sizes keep covering what they are named for."""

# (tokens, dim, wide): the way of fp32, of bf16.  "few": without tiles, by groups of 16 tokens;
# else the tile; "parts": of the sums; "front": tiles of 128 behind those of 256.
FORWARD = [
    ((1, 5441, 8), "few 1 parts", "few 1"),
    ((18, 4190, 9), "few 2 parts", "few 2"),
    ((26, 8134, 8), "few 2 parts", "few 2 parts"),
    ((40, 6400, 100), "few 4 parts", "few 4 parts"),
    ((100, 2500, 200), "single 64 parts", "bf16 64 parts"),
    ((128, 64, 2100), "single 64", "bf16 64"),
    ((925, 7345, 513), "halves 128 parts", "bf16 128 parts"),
    ((524, 23, 13151), "halves 256", "bf16 256"),
    ((1026, 11, 15167), "halves 256 front", "bf16 256 front"),
    ((1473, 2072, 2765), "halves 256 parts", "bf16 128"),
    ((8192, 832, 6400), "halves 256 front", "bf16 256 front"),
]

# The products of the gradients: the tile, and which of dx and dw are in parts; of few tokens
# groups of 16.  fp32, bf16, and bf16 with dw in fp32.
BACKWARD = [
    ((1, 4800, 1600), "few 1 dx", "few 1 dx", "few 1 dx"),
    ((16, 700, 100), "few 1", "few 1", "few 1"),
    ((21, 9, 690), "few 2 dx", "few 2 dx", "few 2 dx"),
    ((30, 1917, 513), "few 2 dx", "few 2 dx", "few 2 dx"),
    ((33, 1601, 255), "few 4", "64", "64"),
    ((63, 130, 5123), "few 4 dx", "64 dx", "64 dx"),
    ((64, 1024, 4096), "few 4 dx", "128 dx", "128 dx"),
    ((827, 8, 545), "64 dx dw", "64 dx dw", "64 dw"),
    ((573, 9, 839), "64 dx dw", "64 dx dw", "64 dx dw"),
    ((4115, 71, 836), "128 dx dw", "128 dx dw", "64 dw"),
    ((1467, 65, 3217), "128 dx dw", "128 dx dw", "128 dx dw"),
    ((4573, 1045, 990), "256 dw", "128 dw", "256 dw"),
    ((1478, 813, 4362), "256 dx dw", "128 dx", "256 dx dw"),
    ((386, 8086, 959), "128", "128", "256"),
    ((5825, 676, 915), "256 dw", "128 dw", "256 dw"),
    ((407, 692, 10427), "256 dx", "128 dx", "256 dx"),
    ((2919, 653, 2807), "256 dx dw", "128", "256 dx dw"),
    ((1401, 3407, 1439), "256", "128", "128"),
    ((129, 1807, 5621), "256 dx", "128 dx", "128 dx"),
    ((3248, 1504, 1195), "256 dw", "256 dw", "256 dw"),
    ((3224, 1893, 975), "256 dw", "256 dw", "256 dw"),
    ((4848, 75, 11246), "256 dx dw", "128 dx dw", "128 dx dw"),
    ((7152, 173, 3259), "256 dx dw", "256 dx dw", "256 dx dw"),
    ((2048, 1600, 1664), "256 dx dw", "128", "128 dw"),
]


def forward_way(size, plan):
    if plan["few"] == "1":
        way = f"few {1 if size[0] <= 16 else 2 if size[0] <= 32 else 4}"
    else:
        way = f"{plan['form']} {plan['tile']}"
    if plan["splits"] != "1":
        return way + " parts"
    if plan["few"] != "1" and plan["tile"] == "256" and int(plan["front"]) < -(-size[2] // 256):
        return way + " front"
    return way


def backward_way(size, plan):
    if plan["back_few"] == "1":
        way = f"few {1 if size[0] <= 16 else 2 if size[0] <= 32 else 4}"
    else:
        way = plan["back_tile"]
    return way + " dx" * (plan["dx_splits"] != "1") + " dw" * (plan["dw_splits"] != "1")
