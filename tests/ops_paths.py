"""Sizes that lead through each kernel of the operators, and what the library's rules
pick for them: test_ops_paths.py holds the rules to it on the CPU, so that the GPU
tests that run these sizes keep covering what they are named for."""

# Cross entropy with gradients by tiles of 256: (tokens, dim, vocab), and whether rows
# take references, how many pieces fp32 and bf16 take.  Columns of dim by whole tiles
# of 256 ("wide": more than 128 of them are wanted), by narrower ones, and both.
GRADIENTS = [
    ((200, 100, 50257), dict(refs=False)),                      # narrow alone
    ((129, 768, 50257), dict(refs=False)),                      # wide alone, three
    ((1030, 129, 50257), dict(refs=False)),                     # wide, one column past the half
    ((1500, 330, 30011), dict(refs=False)),                     # wide and narrow
    ((4100, 64, 30011), dict(refs=True)),                       # narrow alone
    ((2500, 300, 30011), dict(refs=True)),                      # wide and narrow
    ((2304, 768, 50257), dict(refs=True)),                      # wide alone, whole tiles
    ((2051, 1601, 33001), dict(refs=True)),                     # six wide and a narrow one
    ((9000, 129, 65001), dict(refs=True, pieces=(3, 2))),
]

# Losses alone by tiles of 256: whether the last columns of the vocabulary go by 128.
LOSSES = [
    ((1024, 401, 50257), dict(split=True)),
    ((2040, 768, 50257), dict(split=True)),
    ((1500, 100, 30011), dict(split=False)),
    ((4100, 129, 30011), dict(split=False)),
    ((129, 768, 50257), dict(split=False)),
]

# (count, rows, cols): tiles of the symmetric products and of the update.
MATRICES = [
    ((12, 770, 768), (128, 128)),
    ((12, 384, 1152), (64, 128)),
    ((20, 642, 641), (128, 256)),
    ((8, 1025, 1283), (128, 256)),
    ((40, 700, 710), (256, 128)),
    ((64, 385, 389), (256, 256)),
    ((64, 900, 385), (256, 256)),
    ((24, 1023, 1100), (256, 256)),
]
