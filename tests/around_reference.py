"""Plain 64-bit forms of the operators around the attention (norm + rotation +
layout, the 8-bit cache, attention over it), for their tests.  Written from the
definitions in include/vsa2.h with loops and index arithmetic; nothing of the
library runs here."""
import math

import torch

PAGE = 64


# --------------------------------------------------------------------------
# norm, rotation, layout
# --------------------------------------------------------------------------
def place_of(p):
    """For each raster token (grid, then text) its place in the cube-major order,
    and its grid position (None for text)."""
    Nt, Nh, Nw = (-(-n // b) for n, b in ((p.T, p.Bt), (p.H, p.Bh), (p.W, p.Bw)))
    B = p.Bt * p.Bh * p.Bw
    places, where = [], []
    for t in range(p.T):
        for h in range(p.H):
            for w in range(p.W):
                n = ((t // p.Bt) * Nh + h // p.Bh) * Nw + w // p.Bw
                beta = ((t % p.Bt) * p.Bh + h % p.Bh) * p.Bw + w % p.Bw
                places.append(n * B + beta)
                where.append((t, h, w))
    for i in range(p.text_len):
        places.append(Nt * Nh * Nw * B + i)
        where.append(None)
    L = (Nt * Nh * Nw + -(-p.text_len // B)) * B
    return torch.tensor(places), where, L


def turn_of(p, axes, tables, origin, where):
    """cos, sin [batch, tokens, pairs] in 64 bits (rows clamped into the tables)."""
    pairs = sum(axes) // 2
    c = torch.ones(p.batch, len(where), pairs, dtype=torch.float64)
    s = torch.zeros_like(c)
    for b in range(p.batch):
        for i, at in enumerate(where):
            if at is None:
                continue
            first = 0
            for x in range(3):
                n = axes[x] // 2
                if n:
                    row = at[x] + (0 if origin is None else int(origin[b, x]))
                    row = min(max(row, 0), tables[x].shape[0] - 1)
                    c[b, i, first:first + n] = tables[x][row, :, 0].double()
                    s[b, i, first:first + n] = tables[x][row, :, 1].double()
                first += n
    return c, s


def elements_of(pairs, halves):
    i = torch.arange(pairs)
    return (i, i + pairs) if halves else (2 * i, 2 * i + 1)


def turned(x, c, s, halves):
    """x [batch, heads, tokens, D] with its pairs turned by (c, s)."""
    first, second = elements_of(c.shape[-1], halves)
    y = x.clone()
    a, b = x[..., first], x[..., second]
    c, s = c[:, None], s[:, None]
    y[..., first] = a * c - b * s
    y[..., second] = a * s + b * c
    return y


def pair_size(x, pairs, halves):
    """|a| + |b| of the pair each element belongs to (its own size past the pairs)."""
    first, second = elements_of(pairs, halves)
    y = x.abs().clone()
    both = x[..., first].abs() + x[..., second].abs()
    y[..., first] = both
    y[..., second] = both
    return y


def norm_of(x, gain, eps):
    if not eps:
        return x
    u = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return u if gain is None else u * gain


def rope_forward(p, x, gain, eps, cs, halves):
    """(y raster, size of what each element is made of), 64 bits."""
    u = norm_of(x, gain, eps)
    if cs is None:
        return u, u.abs()
    return turned(u, *cs, halves), pair_size(u, cs[0].shape[-1], halves)


def to_places(y, places, L):
    out = torch.zeros(*y.shape[:2], L, y.shape[-1], dtype=y.dtype)
    out[:, :, places] = y
    return out


def rope_backward(x, gain, eps, cs, halves, dy):
    """(dx, dgain, the sizes behind dx, the sizes behind dgain) for raster dy."""
    g, size = dy, dy.abs()
    if cs is not None:
        g, size = turned(dy, cs[0], -cs[1], halves), pair_size(dy, cs[0].shape[-1], halves)
    if not eps:
        return g, None, size, None
    rms = torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    n = x / rms
    w = torch.ones(x.shape[-1], dtype=torch.float64) if gain is None else gain
    h = g * w
    dx = (h - n * (h * n).mean(-1, keepdim=True)) / rms
    behind = (size * w.abs() + n.abs() * (size * w.abs() * n.abs()).mean(-1, keepdim=True)) / rms
    return dx, (g * n).sum((0, 1, 2)), behind, (size * n.abs()).sum((0, 1, 2))


# --------------------------------------------------------------------------
# the cache
# --------------------------------------------------------------------------
def e4m3_values():
    """Value of each of the 256 codes (NaN for 0x7f and 0xff)."""
    v = []
    for code in range(256):
        sign, e, m = -1.0 if code & 128 else 1.0, (code >> 3) & 15, code & 7
        if e == 15 and m == 7:
            v.append(math.nan)
        else:
            v.append(sign * (math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)))
    return torch.tensor(v, dtype=torch.float64)


VALUES = e4m3_values()


def e4m3_codes(y):
    """Nearest code of each value (|y| <= 448), ties to the even code."""
    grid = VALUES[:127]                       # 0 .. 448 ascending
    a = y.abs()
    hi = torch.searchsorted(grid, a.contiguous()).clamp(1, 126)
    lo = hi - 1
    up, down = grid[hi] - a, a - grid[lo]
    code = torch.where(up < down, hi, torch.where(up > down, lo, torch.where(hi % 2 == 0, hi, lo)))
    code = torch.where(a == 0, torch.zeros_like(code), code)
    return code + 128 * torch.signbit(y)


def quantised(x):
    """(codes, powers) of rows x [..., D]; values that are not finite get code 0x7f."""
    x = x.double()
    fine = torch.isfinite(x)
    top = torch.where(fine, x.abs(), 0.0).amax(-1)
    e = torch.full(top.shape, -100, dtype=torch.int64)
    for k in range(-100, 121):
        e = torch.where(top > 448.0 * 2.0 ** k, k + 1, e)
    y = torch.where(fine, x, 0.0) * torch.pow(2.0, -e.double())[..., None]
    return torch.where(fine, e4m3_codes(y), 0x7f), e


def offsets(j, D):
    """Byte offsets in a page of token j: K codes [D], V codes [D], K power, V power."""
    t, r, g, i = j // 16, j % 16, (j // 4) % 4, j % 4
    e = torch.arange(D)
    k = ((t * (D // 64) + e // 64) * 64 + (e % 64) // 16 * 16 + r) * 16 + e % 16
    v = 64 * D + ((e // 16) * 64 + g * 16 + e % 16) * 16 + t * 4 + i
    return k, v, 128 * D + r * 4 + t, 128 * D + 64 + g * 16 + t * 4 + i


def page_for(table, b, h, pos, pages):
    """Page of list position pos for KV head h, or None."""
    lists = table[b] if table.dim() == 2 else table[b, h]
    if pos < 0 or pos >= lists.shape[0] * PAGE:
        return None
    page = int(lists[pos // PAGE])
    return page if 0 <= page < pages else None


def write_reference(pool, table, k, v, start, count):
    """pool (CPU, changed in place) after the write of k, v [batch, heads, n, D]."""
    D = k.shape[-1]
    codes = [quantised(x) for x in (k, v)]
    for b in range(k.shape[0]):
        for i in range(min(k.shape[2], int(count[b]) if count is not None else k.shape[2])):
            for h in range(k.shape[1]):
                pos = int(start[b]) + i
                page = page_for(table, b, h, pos, pool.shape[0])
                if page is None:
                    continue
                places = offsets(pos % PAGE, D)
                for x in range(2):
                    pool[page, h, places[x]] = codes[x][0][b, h, i].to(torch.uint8)
                    pool[page, h, places[2 + x]] = int(codes[x][1][b, h, i]) + 127
    return pool


def token_values(pool, table, b, h, pos, D):
    """(k, v) [D] in 64 bits of one list position, or None."""
    page = page_for(table, b, h, pos, pool.shape[0])
    if page is None:
        return None
    at = offsets(pos % PAGE, D)
    row = pool[page, h]
    return tuple(VALUES[row[at[x]].long()] * 2.0 ** (int(row[at[2 + x]]) - 127) for x in range(2))


def read_reference(pool, table, n, start, count, D, heads):
    k = torch.zeros(2, table.shape[0], heads, n, D, dtype=torch.float64)
    for b in range(table.shape[0]):
        for i in range(min(n, int(count[b]) if count is not None else n)):
            for h in range(heads):
                x = token_values(pool, table, b, h, int(start[b]) + i, D)
                if x is not None:
                    k[0, b, h, i], k[1, b, h, i] = x
    return k[0], k[1]


def attn_reference(pool, table, q, length, count, causal):
    """(o, lse, sum p |v|, largest sum |q k| / sqrt(D)) of q [batch, heads, n, D]."""
    b_, hq, n, D = q.shape
    heads = pool.shape[1]
    group = hq // heads
    o = torch.zeros(b_, hq, n, D, dtype=torch.float64)
    lse = torch.full((b_, hq, n), -math.inf, dtype=torch.float64)
    weight = torch.zeros_like(o)
    logit = torch.zeros(b_, hq, n, 1, dtype=torch.float64)
    for b in range(b_):
        cnt = n if count is None else min(max(int(count[b]), 0), n)
        total = min(max(int(length[b]), 0), table.shape[-1] * PAGE)
        for h in range(heads):
            rows = {pos: token_values(pool, table, b, h, pos, D) for pos in range(total)}
            for i in range(cnt):
                limit = total - (cnt - 1 - i) if causal else total
                seen = [rows[pos] for pos in range(max(0, limit)) if rows[pos] is not None]
                if not seen:
                    continue
                k, v = torch.stack([x[0] for x in seen]), torch.stack([x[1] for x in seen])
                for y in range(h * group, (h + 1) * group):
                    s = k @ q[b, y, i].double() / math.sqrt(D)
                    lse[b, y, i] = torch.logsumexp(s, 0)
                    w = torch.softmax(s, 0)
                    o[b, y, i] = w @ v
                    weight[b, y, i] = w @ v.abs()
                    logit[b, y, i] = (k.abs() @ q[b, y, i].double().abs()).max() / math.sqrt(D)
    return o, lse, weight, logit
