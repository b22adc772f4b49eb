"""How the norms' backward call adds over the tokens (tests/test_norm_plans.py holds `groups` to the library's plan)."""


def groups(T, d):
    """Groups of threads, each of which takes every groups-th row: those of 64 threads come in fours."""
    up = lambda a, b: -(-a // b)
    if d <= 512:
        return min(512, up(T, 4)) * 4
    return min(1024 if d <= 2048 else 512 if d <= 4096 else 256, max(up(T, 2), min(T, 128)))


def chain(T, d):
    """The longest chain of additions of a sum over the tokens: a group's rows, every sixteenth group by a thread, 16 threads."""
    g = groups(T, d)
    return -(-T // g) + -(-g // 16) + 16
