"""Calls that reach every kernel of the products with group scales (CPU: checked with the library's own plans; GPU: run).
(fp32 tokens, gated, group, T, n_in, n_out)"""
KINDS = ((128, 384), (64, 384), (32, 384), (96, 288))   # a scale a window, two, four, any other group


def _cases():
    for xf32 in (0, 1):
        for gated in (0, 1):
            for n_out in (100, 8500, 17000):              # 8, 4 and 2 waves to a row tile
                yield xf32, gated, 64, 1, 544 * 2, n_out
                for group, n_in in KINDS:
                    yield xf32, gated, group, 2, n_in, n_out
            for k, (group, n_in) in enumerate(KINDS):
                long = 32 * 288 if k == 3 else 8192       # rows whose x does not fit in LDS at once
                yield xf32, gated, group, 4 if xf32 else 16, long, 40
                if xf32:
                    yield xf32, gated, group, 16, long, 40
                for T in (20, 40, 60):
                    yield xf32, gated, group, T, n_in, 150
            # rows in shares: one token, one tile, three; x of one token in pieces
            yield xf32, gated, 128, 1, 32768, 64
            yield xf32, gated, 64, 3, 16384, 64
            yield xf32, gated, 32, 40, 2048, 64
            yield xf32, gated, 128, 1, 36864, 8192


CASES = list(_cases())
