"""How the embedding's gradient is divided: sizes of the pieces that sorted tokens are cut into, and how many roundings a term passes for it."""


def pieces(n, dim):
    """Tokens of a piece, and their number: pieces of 8, doubled while there are more than 2048 for every 512 columns (512 at least)."""
    most, piece = max(512, 2048 // -(-dim // 512)), 8
    while -(-n // piece) > most:
        piece *= 2
    return piece, -(-n // piece)


def roundings(n, dim):
    """Most additions that a token's row passes, and the product.  A wave adds a piece and up to 8 tokens behind it, one after another; 16 waves add a share each of
    the pieces of an id, one after another, and 4 halvings join them."""
    piece, count = pieces(n, dim)
    return min(n, piece + 8) + -(-count // 16) + 4 + 1


def workspace_bytes(n, vocab, dim):
    up = lambda b: -(-b // 256) * 256
    tile = -(-max(1024, -(-n // 64)) // 256) * 256
    count = pieces(n, dim)[1]
    return 4 * up(4 * n) + up(-(-n // tile) * 512 * 4) + up(count * 2 * dim * 4) + up((count + 1) * 4)
