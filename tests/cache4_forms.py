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

KINDS = ("few", "fp32", "many")                      # 16 bf16 rows, 16 fp32 rows, 32 bf16 rows together


def form(kind, d, runs, page=16, **more):
    """A small case of one form: by its rows, its channels, and blocks per unit or (in tables wide enough) runs."""
    c = dict(lengths=[(29 * b) % 80 + (b > 0) for b in range(6)], N=3, Hq=4, H=2, dtype=F32 if kind == "fp32" else BF16)
    if kind == "many":
        c.update(lengths=[(29 * b) % 80 + (b > 0) for b in range(22)], N=60, Hq=8, H=2)
    return dict(c, d=d, page=page, entries=(17408 if runs else 512) // page, **more)


def nan_lengths(kind):
    """Longer ones, so that runs cut the units of many samples: up to 500 entries."""
    return [40 + (67 * b) % (190 if kind == "many" else 461) for b in range(22 if kind == "many" else 6)]


FORMS = [(kind, d, runs) for kind in KINDS for d in (64, 128) for runs in (0, 1)]

# Joins: fp32 rows of 128 and of 64 channels in runs, a block per row and per sixteen rows (more than 2048 rows in the call)
JOINS = [
    dict(lengths=[0, 700, 1, 33, 0, 1234, 64], N=3, Hq=4, H=2, d=128, page=16, dtype=F32, entries=200, keep=0.6),
    dict(lengths=[300, 40, 90], N=90, Hq=12, H=2, d=128, page=256, dtype=F32, entries=65, q_len=[90, 41, 90]),
    dict(lengths=[300, 40, 90], N=90, Hq=12, H=2, d=64, page=256, dtype=F32, entries=65, q_len=[90, 41, 90]),
    dict(lengths=[(29 * b) % 80 for b in range(22)], N=20, Hq=13, H=13, d=64, page=256, dtype=BF16, entries=65, keep=0.8),
]
# One long sample among short ones: parts of one row by the hundred, few waves to a row
LONG = dict(lengths=[43211] + [1 + (11 * b) % 60 for b in range(40)], N=1, Hq=1, H=1, page=64, entries=700)


def parts_of(lengths, N, Hq, H, rows, blocks=1024, least=4):
    """Parts of the first sample's first unit in runs of equal work."""
    steps = [max(1, -(-n // 32)) for n in lengths]
    tiles = -(-N * (Hq // H) // rows)
    total = sum(H * tiles * s for s in steps)
    runs = min(max(total // least, 1), blocks)
    return (steps[0] * runs - 1) // total + 1
