"""Which kernel multiplies matrices in 8 bits, as the library chooses: tests of one of the two ask here whether their sizes reach it, and
test_packed_paths.py holds what is said here to the library's workspaces."""
BLOCK = 128
CUT_FROM = 24  # blocks of columns from which tiles that leave compute units idle are cut along K

SHORT = 5      # blocks of a row of h up to which tiles note elements near ties of two codes


def blocks(n):
    return -(-n // BLOCK)


def takes_tiles(rows, groups, N, K, activation=False):
    """Whether the product of `rows` rows of `groups` groups with matrices [N][K] runs in tiles; `activation`: the experts' first product."""
    if K <= BLOCK or rows <= (64 if groups == 1 else 48) * groups:
        return False
    stretches = -(-rows // 64) if groups == 1 else (rows + 32 * groups) // 64
    workgroups = stretches * -(-N // (128 if activation else 64))
    return workgroups > (384 if activation else 512) or workgroups * K > (1 << 20 if activation else 1 << 21)


def experts_take_tiles(T, d, f, S, k):
    """(the first product, the second)"""
    return takes_tiles(T * k, S, f, d, True), takes_tiles(T * k, S, d, f)


def converts_its_rows(rows, K):
    """Whether a streaming product converts the rows itself."""
    return rows <= 16 and rows * blocks(K) <= 128
