"""Calls of the head's losses under a limit of the workspace, and what becomes of their pieces' gradients of W (tests/test_head_workspace.py
checks that): tokens, vocabulary, width, fp32, limit in bytes."""
PIECES = {
    "runs of K": (5000, 500, 264, False, 6_000_000),
    "256-wide, the last round in quarters": (9000, 8200, 2056, False, 130_000_000),
    "256-wide": (3000, 9067, 1032, False, 60_000_000),
    "fp32, runs of K": (6000, 1500, 264, True, 60_000_000),
}
