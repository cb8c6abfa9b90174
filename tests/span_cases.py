"""Calls that reach every row-block shape of attention under a window and over a 4-bit
cache with little work for an oracle: a few short sequences in a large padded batch of
tokens, or few different sequences of a verification many times over.  The shapes that
the plan gives them on 256 compute units are checked on the CPU
(tests/test_span_shapes_host.py)."""

# (new, kv): blocks of every size end inside a sequence; one fits its cache, one has none
# new, and one has tokens before its first position, which see nothing.
LENS = [(60, 350), (1, 300), (17, 20), (33, 33), (0, 40), (20, 7)]
NEW = sum(n for n, _ in LENS)
HEADS = [(16, 2), (15, 1)]
TOKENS = [NEW, 1000, 2000, 3000, 4000, 8000, 16000]
# window, sinks, mask_block
WINDOWS = [(100, 12, 1), (40, 70, 8), (1, 0, 1), (345, 0, 4)]
WHOLE = [(0, 0, 1), (0, 0, 8), (0, 0, 0)]                      # (4 bits only: the others are the call without one)

PREFIXES = [300, 0, 97]
STEPS = [(8, 8, 32, 2), (32, 32, 8, 2), (7, 4, 15, 1)]         # block, references, heads
COPIES = [1, 16, 32, 64, 128]

SHAPES = {"bf16": {64, 128, 256}, "fp4": {32, 64, 128, 256}, "f32": {16, 32, 64, 128}}


def windows(form):
    return WINDOWS + (WHOLE if form == "fp4" else [])
