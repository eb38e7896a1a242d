"""Plain 64-bit (or whole-number) implementations of token sampling, rotary positions, the book of a cache's pages and cross attention (imported by
test files; not a test module).  numpy on the host; nothing here uses the library."""
import numpy as np

from lm_util import F, U, to_np

EMPTY = (-1, -1, 0)


# ---- token sampling -----------------------------------------------------------------------------
def sample_reference(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(id, logprob, near): near where the draw or a limit lies so close to a border that the rounding of weights to whole numbers may decide."""
    x = np.asarray(x, np.float64)
    if not (0 <= temperature < np.inf) or np.isnan(top_p) or np.isnan(min_p) or not 0 <= u < 1:
        return -1, np.nan, False
    if np.isnan(x).any() or x.max() in (np.inf, -np.inf):
        return -1, np.nan, False
    order = np.argsort(-x, kind="stable")
    if temperature == 0 or min_p > 1:
        return int(order[0]), 0.0, False
    with np.errstate(over="ignore"):
        w = np.exp((x - x.max()) / temperature)
    # a weight is off by half a unit of 2^-s at most (s = 46, or 62 less the bits of the vocabulary), and by 2^-48 of itself for exponential and argument
    unit = 2.0 ** -min(46, 62 - int(np.ceil(np.log2(len(x) + 1))))
    slack = len(x) * unit + 2.0 ** -40 * w.sum()
    sums, m, near = np.cumsum(w[order]), len(x), False
    if top_k > 0:
        m = min(m, top_k)
    if top_p < 1:
        target = top_p * w.sum()
        reached = int(np.searchsorted(sums, target, side="left")) + 1
        if reached <= m:                                        # (equal weights are whole numbers of one size: their sums are exact)
            near |= len(set(w)) > 1 and np.abs(sums - target).min() < slack
            m = reached
    m = max(1, min(m, int((w >= min_p).sum())))
    kept = np.zeros(len(x))
    kept[order[:m]] = w[order[:m]]
    mass = np.cumsum(kept)
    at = u * mass[-1]
    token = int(np.searchsorted(mass, at, side="right"))
    near |= len(set(kept) - {0.0}) > 1 and np.abs(mass - at).min() < slack and u > 0
    return token, np.log(kept[token] / mass[-1]), near


def sample_bound(logprob):
    """The result's own rounding; weights and their sum, off by 2^-28 relative at most; angles and logarithms are in 64 bits."""
    return F * abs(logprob) + 2.0 ** -27


# ---- rotary positions ---------------------------------------------------------------------------
def rotate_reference(x, positions, frequencies, sections, neighbours, inverse):
    x = to_np(x)
    pos = to_np(positions).reshape(x.shape[0], -1)
    f = to_np(frequencies)
    half = len(f)
    axis = np.repeat(np.arange(len(sections)), sections)
    angle = pos[:, axis] * f * (-1 if inverse else 1)
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if neighbours else (slice(0, half), slice(half, 2 * half))
    out = x.copy()
    out[..., first] = x[..., first] * cos - x[..., second] * sin
    out[..., second] = x[..., first] * sin + x[..., second] * cos
    size = np.abs(x)
    size[..., first] = size[..., second] = np.abs(x[..., first]) + np.abs(x[..., second])
    size[..., 2 * half:] = 0
    return out, size


def rotate_bound(out, size, bf16, turns):
    """The output's own rounding; two products and a sum in fp32, sine and cosine good to two units (2^-23) and their fraction of a turn to 2^-25 of at
    most half a turn, pi in radians: 2^-23; and the whole turns, formed with three roundings of 2^-53."""
    return (U if bf16 else F) * np.abs(out) + (8 * F + turns * 2.0 ** -48) * size


# ---- the book of a cache's pages ----------------------------------------------------------------
class Book:
    """mt_kv_pages, restated with lists.  Every call returns its errors as (code, index)."""

    def __init__(self, refs, tables, lengths, page):
        self.refs, self.tables, self.lengths, self.page = list(refs), [list(t) for t in tables], list(lengths), page

    def good(self, row):
        return 0 <= row < len(self.lengths) and 0 <= self.lengths[row] <= len(self.tables[row]) * self.page

    def held(self, row):
        return self.tables[row][: -(-self.lengths[row] // self.page)]

    def free(self):
        return [i for i, r in enumerate(self.refs) if r <= 0]

    def reserve(self, rows, counts, n_slots):
        free, taken, at, errors = self.free(), 0, 0, []
        slots = [-1] * n_slots
        for i, (r, c) in enumerate(zip(rows, counts)):
            ok = r not in rows[:i] and self.good(r) and c >= 0 and self.lengths[r] + c <= len(self.tables[r]) * self.page
            code, need, first, c = 1, 0, at, max(c, 0)
            at += c
            if ok:
                had = -(-self.lengths[r] // self.page)
                need = -(-(self.lengths[r] + c) // self.page) - had
                if need and taken + need > len(free):
                    ok, code = False, 5
                elif first + c > n_slots:
                    ok = False
                else:
                    for j in range(need):
                        self.tables[r][had + j] = free[taken + j]
                        self.refs[free[taken + j]] = 1
                    for j in range(c):
                        t = self.lengths[r] + j
                        slots[first + j] = self.tables[r][t // self.page] * self.page + t % self.page
                    self.lengths[r] += c
            if not ok:
                errors.append((code, i))
            taken += need
        return slots, errors

    def fork(self, parents, children):
        free, taken, copies, errors, changes = self.free(), 0, [], [], []
        for i, (p, c) in enumerate(zip(parents, children)):
            copy = EMPTY
            ok = self.good(p) and self.good(c) and c not in children[:i] and all(0 <= x < len(self.refs) for x in self.held(p))
            if not ok:
                errors.append((1, i))
            elif p != c:
                part = self.lengths[p] % self.page
                row = list(self.held(p))
                if part and taken >= len(free):
                    errors.append((5, i))
                else:
                    if part:
                        copy = (row[-1], free[taken], part)
                        row[-1] = free[taken]
                    changes.append((i, c, row, self.lengths[p], bool(part)))
                taken += bool(part)
            copies.append(copy)
        old = {c: list(self.held(c)) for _, c, _, _, _ in changes}
        for i, c, row, n, part in changes:
            for x in row[: len(row) - part]:
                self.refs[x] += 1
            if part:
                self.refs[row[-1]] = 1
            for x in old[c]:
                self.refs[x] -= 1
            self.tables[c][: len(row)] = row
            self.lengths[c] = n
        return copies, errors

    def release(self, rows):
        errors = []
        for i, r in enumerate(rows):
            if r in rows[:i] or not self.good(r):
                errors.append((1, i))
                continue
            for x in self.held(r):
                self.refs[x] -= 1
            self.lengths[r] = 0
        return errors

    def compact(self, most):
        used = sum(r > 0 for r in self.refs)
        holes = [i for i, r in enumerate(self.refs) if r <= 0 and i < used]
        high = [i for i, r in enumerate(self.refs) if r > 0 and i >= used]
        to = dict(list(zip(high, holes))[:most])
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        for r in range(len(self.lengths)):
            if self.good(r):
                n = len(self.held(r))
                self.tables[r][:n] = [to.get(x, x) for x in self.tables[r][:n]]
        return ([(a, b, self.page) for a, b in to.items()] + [EMPTY] * most)[:most]


# ---- cross attention ----------------------------------------------------------------------------
def cross_reference(q, k, v, offsets, ranges, scale):
    """(o, a): outputs, and sum p |v|.  NaN where no sequence writes."""
    q, k, v = to_np(q), to_np(k), to_np(v)
    g = q.shape[1] // k.shape[1]
    o, a = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for s, (lo, hi) in enumerate(zip(offsets[:-1], offsets[1:])):
        first, end = ranges[s]
        if hi <= lo:
            continue
        if end == first:
            o[lo:hi] = a[lo:hi] = 0
            continue
        for h in range(q.shape[1]):
            z = q[lo:hi, h] @ k[first:end, h // g].T * scale
            p = np.exp(z - z.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o[lo:hi, h] = p @ v[first:end, h // g]
            a[lo:hi, h] = p @ np.abs(v[first:end, h // g])
    return o, a
