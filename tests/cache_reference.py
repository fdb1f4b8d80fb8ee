"""The 8-bit paged K/V cache and the attention over it, in 64 bits and one element at a time where order matters: what include/hgf.h says, written
apart from the library.  Tensors are CPU numpy arrays; K, V and Q come as bf16 bit patterns (uint16)."""
import numpy as np

from paper_2602_05269_b200.inputs import bf16_bits_to_f32, f32_to_bf16_bits

BLOCK = 64


def tile_index(rows, cols):
    """[rows][cols] -> byte of each element: tiles of 16 x 32, byte (4 g + t) * 16 + 8 h + 4 a + b of a tile."""
    r, c = np.meshgrid(np.arange(rows), np.arange(cols), indexing="ij")
    return ((r // 16) * (cols // 32) + c // 32) * 512 + (4 * (r % 8) + c // 4 % 4) * 16 + 8 * (c // 16 % 2) + 4 * (r // 8 % 2) + c % 4


def page_bytes(k1, k2, v):
    """Codes [64][dh] of K1, K2, V -> the 3 * 64 * dh bytes that a page holds for a head."""
    dh = k1.shape[1]
    out = np.zeros(3 * BLOCK * dh, np.int8)
    for n, x in enumerate((k1, k2, v.T)):
        out[n * BLOCK * dh + tile_index(*x.shape)] = x
    return out


def quantise(x):
    """x [64][dh] float64 of one head -> (codes, scale as binary32): Round(127 x / max |x|), max |x| / 127."""
    top = np.abs(x).max()
    if not np.isfinite(x).all():
        return np.zeros(x.shape, np.int8), np.float32(np.nan)
    if top == 0:
        return np.zeros(x.shape, np.int8), np.float32(0)
    return np.rint(127 * x / top).astype(np.int8), np.float32(np.float32(top) / np.float32(127))


class Reference:
    """Sequences as lists of tokens; pages and counts as the calls deal them."""

    def __init__(self, H, dh, n_pages, n_slots, max_pages):
        self.H, self.dh, self.n_pages, self.max_pages = H, dh, n_pages, max_pages
        self.tokens = [[] for _ in range(n_slots)]   # bf16 bits [3][H][dh] of each token
        self.pages = [[] for _ in range(n_slots)]    # page numbers held
        self.refs = [0] * n_pages
        self.content = {}                            # page -> (codes [3][H][64][dh], scales [3][H])

    def reserve(self, slots, tokens):
        free, seen, granted, short = [p for p in range(self.n_pages) if not self.refs[p]], set(), [], False
        for s, t in zip(slots, tokens):
            if not 0 <= s < len(self.tokens) or s in seen or t // BLOCK > self.max_pages:
                granted.append(0)
                seen.add(s)
                continue
            seen.add(s)
            need = max(0, t // BLOCK - len(self.pages[s]))
            short = short or need > len(free)
            if need and short:
                granted.append(0)
                continue
            for p in free[:need]:
                self.refs[p] = 1
                self.pages[s].append(p)
            free = free[need:]
            granted.append(1)
        return granted

    def append(self, slots, starts, k, v):
        """k, v: bf16 bits [n][2 H dh], [n][H dh]."""
        seen, done = set(), []
        for i, s in enumerate(slots):
            rows = range(starts[i], starts[i + 1])
            ok = 0 <= s < len(self.tokens) and s not in seen
            seen.add(s)
            if ok:
                n0, n1 = len(self.tokens[s]), len(self.tokens[s]) + len(rows)
                ok = n1 // BLOCK <= len(self.pages[s]) and all(self.refs[p] == 1 for p in self.pages[s][n0 // BLOCK:n1 // BLOCK])
            done.append(int(ok))
            if not ok:
                continue
            for r in rows:
                self.tokens[s].append(np.concatenate([k[r].reshape(2, self.H, self.dh), v[r].reshape(1, self.H, self.dh)]))
            for b in range(n0 // BLOCK, n1 // BLOCK):
                x = bf16_bits_to_f32(np.stack(self.tokens[s][b * BLOCK:(b + 1) * BLOCK])).astype(np.float64)
                q = [[quantise(x[:, n, h]) for h in range(self.H)] for n in range(3)]
                self.content[self.pages[s][b]] = (np.stack([[c for c, _ in row] for row in q]), np.array([[sc for _, sc in row] for row in q], np.float32))
        return done

    def fork(self, src, dst):
        done = []
        for i, (a, b) in enumerate(zip(src, dst)):
            ok = all(0 <= x < len(self.tokens) for x in (a, b)) and b not in dst[:i] and a not in dst and not self.tokens[b] and not self.pages[b]
            done.append(int(ok))
            if ok:
                self.tokens[b] = list(self.tokens[a])
                self.pages[b] = self.pages[a][:len(self.tokens[a]) // BLOCK]
                for p in self.pages[b]:
                    self.refs[p] += 1
        return done

    def free(self, slots):
        for s in dict.fromkeys(slots):
            if 0 <= s < len(self.tokens):
                for p in self.pages[s]:
                    self.refs[p] -= 1
                self.tokens[s], self.pages[s] = [], []

    def values(self, s):
        """K1, K2, V [H][length][dh] in 64 bits that the cache stands for."""
        n = len(self.tokens[s])
        out = np.zeros((3, self.H, n, self.dh))
        for b in range(n // BLOCK):
            codes, scales = self.content[self.pages[s][b]]
            out[:, :, b * BLOCK:(b + 1) * BLOCK] = codes.astype(np.float64) * scales[:, :, None, None].astype(np.float64)
        if n % BLOCK:
            out[:, :, n // BLOCK * BLOCK:] = bf16_bits_to_f32(np.stack(self.tokens[s][n // BLOCK * BLOCK:])).astype(np.float64).transpose(1, 2, 0, 3)
        return out


def attention(values, q, m, heads, lam, out_scale, coarse=False):
    """values [3][H][n][dh]; q float64 [m][2][heads][dh], the last m of n tokens -> (out [m][heads][dh], tolerance of each row and head).

    The tolerance follows the kernel's number formats: q to 2^-22 of its row's largest magnitude (a score is off by that times the sum of |k|), scores and
    exponentials in binary32 (four roundings of the score's size, 2^-22 of the exponential; a score's absolute error is a probability's relative
    one, twice with the normalisation), probabilities to 2^-24 of the largest (twice that, with what the sum has left of it), sums of one term a page in
    binary32; all of it times the largest |v| and both streams' weights.  `coarse`: probabilities to 2^-17 of the largest in their page of 64, so a page's
    are off by 64 * 2^-17 of its largest at most, which is no more than its weight: all of them by 2^-11 of the sum."""
    _, H, n, dh = values.shape
    out, tol = np.zeros((m, heads, dh)), np.zeros((m, heads))
    for j in range(m):
        sees = n - m + j + 1
        if sees <= 0:
            continue
        for h in range(heads):
            kv = values[:, h // (heads // H), :sees]
            big = np.abs(kv[2]).max()
            for st, w in ((0, 1.0), (1, lam)):
                s = kv[st] @ q[j, st, h] / np.sqrt(dh)
                p = np.exp(s - s.max())
                out[j, h] += w * (1 if st == 0 else -1) * (p @ kv[2]) / p.sum()
                ds = 2.0 ** -22 * np.abs(q[j, st, h]).max() * np.abs(kv[st]).sum(1).max() / np.sqrt(dh) + 4 * 2.0 ** -24 * np.abs(kv[st] * q[j, st, h]).sum(1).max() / np.sqrt(dh)
                tol[j, h] += abs(w) * big * (2 * (ds + 2.0 ** -21) + 2 * sees * 2.0 ** -24 / p.sum() + (sees / BLOCK + 20) * 2.0 ** -23 + (2.0 ** -11 if coarse else 0))
    return out * out_scale, tol * abs(out_scale)


def rows(rng, n, width, spread=1.0):
    return f32_to_bf16_bits((rng.standard_normal((n, width)) * spread).astype(np.float32))
