"""Sizes that the projections' kernel of 256 x 256 tiles takes."""


def tile_size(sms, width=128):
    """Rows and features, a multiple of 4 that ends inside a tile, whose 128 x
    `width` tiles are more than two thirds of the SMs."""
    rows = 1300
    down = (rows + 127) // 128
    across = (2 * sms // 3) // down + 2
    return rows, width * across - 36
