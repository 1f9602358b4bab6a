"""Cases of the attention over the cache held in 4 bits, by the form that they take (test infrastructure)."""
BF16, F32 = "bf16", "f32"

# 32 query rows together: blocks per unit, runs; drafts of four tokens of a batch that is just large enough for it
MANY_ROWS = [
    dict(lengths=[(29 * b) % 80 for b in range(22)], N=20, Hq=13, H=13, d=64, page=32, dtype=BF16, entries=16),
    dict(lengths=[(29 * b) % 80 for b in range(22)], N=20, Hq=13, H=13, d=128, page=32, dtype=BF16, entries=16),
    dict(lengths=[(29 * b) % 80 for b in range(22)], N=20, Hq=13, H=13, d=64, page=256, dtype=BF16, entries=65),
    dict(lengths=[(29 * b) % 80 for b in range(22)], N=20, Hq=13, H=13, d=128, page=256, dtype=BF16, entries=65),
    dict(lengths=[20 + (17 * b) % 60 for b in range(33)], N=4, Hq=64, H=8, d=128, page=16, dtype=BF16, entries=8),
]
