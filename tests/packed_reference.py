"""Plain forms of the paged 4-bit cache in numpy and 64 bits, written from the format's description: a sequential page allocator, the
quantiser by search over all representable numbers, tiles taken apart byte by byte."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# the non-negative finite e4m3 numbers by their bits (the index is the byte)
SCALES = np.array([(8 + b % 8) * 2.0 ** (b // 8 - 10) if b >= 8 else b * 2.0 ** -9 for b in range(127)])


def nearest(y, grid):
    """Index of the grid point nearest to y >= 0, halfway the even index, past the end the last one."""
    up = np.clip(np.searchsorted(grid, y), 1, len(grid) - 1)
    below, above = y - grid[up - 1], grid[up] - y
    return np.where((below < above) | ((below == above) & ((up - 1) % 2 == 0)), up - 1, up)


def quantise(x):
    """x [..., d] in 64 bits -> codes [..., d] (sign in bit 3), scale bytes [..., d/16]."""
    g = x.reshape(*x.shape[:-1], -1, 16)
    top = np.clip(np.abs(g).max(-1), 6 * 2.0 ** -9, 6 * 448.0)
    scale = nearest(top, 6 * SCALES)
    s = SCALES[scale][..., None]
    code = np.empty(g.shape, np.int64)
    flat_g, flat_s, flat_c = np.abs(g).reshape(-1, 16), s.reshape(-1), code.reshape(-1, 16)
    for sv in np.unique(flat_s):  # a grid for each scale: no quotient is rounded
        rows = flat_s == sv
        flat_c[rows] = nearest(np.minimum(flat_g[rows], 6 * sv), sv * MAGNITUDES)
    return (flat_c.reshape(x.shape) + 8 * np.signbit(x)), scale


def dequantise(codes, scale):
    v = MAGNITUDES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    return v * np.repeat(SCALES[scale], 16, axis=-1)


def pack(kc, vc, ks, vs):
    """Codes [16, d] and scale bytes [16, d/16] of K and V of 16 tokens of one head -> the tile's 18 d bytes."""
    d = kc.shape[1]
    n, w = d // 16, d // 64
    out = np.zeros(18 * d, np.uint8)
    for u in range(16):
        h, k = u // 8, u % 8
        for e in range(0, d, 2):
            out[u * d // 2 + e // 2] = kc[u, e] | kc[u, e + 1] << 4
            c, b = e // (d // 8), (e % (d // 8)) // 2
            out[8 * d + ((h * 8 + c) * 8 + k) * n + b] = vc[u, e] | vc[u, e + 1] << 4
        for i in range(n):
            out[16 * d + k * 2 * n + (i // w) * 2 * w + h * w + i % w] = ks[u, i]
            out[17 * d + i * 16 + (k // 2) * 4 + h * 2 + k % 2] = vs[u, i]
    return out


class Allocator:
    """The page table rules, one sequence after another."""

    def __init__(self, num_pages, page_len, num_seqs, max_pages):
        self.num_pages, self.P, self.n, self.most = num_pages, page_len, num_seqs, max_pages

    def release(self, finished, lens, table, free, count):
        free, lens = free.copy(), lens.copy()
        for r in range(self.n):
            if finished[r]:
                for j in range(-(-lens[r] // self.P)):
                    if count < self.num_pages:
                        free[count] = table[r, j]
                        count += 1
                lens[r] = 0
        return lens, free, count

    def assign(self, lens, new, table, free, count, max_rows):
        lens, table = lens.copy(), table.copy()
        slots, positions = np.full(max_rows, -1, np.int32), np.zeros(max_rows, np.int32)
        start = [0]
        asked = 0  # pages of all sequences up to here that fit their rows of the table
        left = count
        for r in range(self.n):
            row = start[-1]
            start.append(row + new[r])
            have = -(-lens[r] // self.P)
            fits = lens[r] + new[r] <= self.most * self.P
            need = -(-(lens[r] + new[r]) // self.P) - have if fits else 0
            asked += need
            granted = fits and row + new[r] <= max_rows and (need == 0 or asked <= count)
            if granted:
                for j in range(need):
                    left -= 1
                    table[r, have + j] = free[left]
            for i in range(new[r]):
                if row + i >= max_rows:
                    break
                pos = lens[r] + i
                positions[row + i] = pos
                if granted:
                    slots[row + i] = table[r, pos // self.P] * self.P + pos % self.P
            if granted:
                lens[r] += new[r]
        return lens, table, left, np.array(start, np.int32), slots, positions
