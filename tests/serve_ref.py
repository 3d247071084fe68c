"""Plain 64-bit forms of rotary positions, the 8-bit cache and windowed attention, and layouts
to try them on.  Torch on the device it is given; no call of the library."""
import math

import torch

BS = 16


def pow2(e):
    """2^e in 64 bits, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def rotate(x, pos, freq, pairs, amplitude=1.0):
    """x [rows, heads, d] at positions pos [rows]; freq float64 [R / 2]; pairs 0: halves, 1: neighbours."""
    y, R = x.double().clone(), 2 * freq.shape[0]
    t = pos.double()[:, None, None] * freq
    c, s = torch.cos(t) * amplitude, torch.sin(t) * amplitude
    a, b = (slice(0, R // 2), slice(R // 2, R)) if pairs == 0 else (slice(0, R, 2), slice(1, R, 2))
    x0, x1 = x[..., a].double(), x[..., b].double()
    y[..., a], y[..., b] = x0 * c - x1 * s, x1 * c + x0 * s
    return y


def exponent(x):
    """The smallest e >= -110 with max|x| <= 448 * 2^e, along the last dimension."""
    m, e = torch.frexp(x.double().abs().amax(-1))
    return torch.where(m > 0, e - 9 + (m > 0.875), -110).clamp(min=-110)


def e4m3(y):
    """y (|y| <= 448) rounded to the nearest e4m3 number, ties to even."""
    ulp = pow2(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(y / ulp) * ulp


def quantise(x):
    """(values that x [..., d] is stored as, its power's byte [...])."""
    e = exponent(x)
    step = pow2(e)[..., None]
    return e4m3(x.double() / step) * step, (e + 127).to(torch.uint8)


def visible(pos, keys, window, sinks):
    """[rows, keys]: whether the row at pos sees key j."""
    p, j = pos[:, None], torch.arange(keys, device=pos.device)[None, :]
    seen = j <= p
    if window:
        seen = seen & ((j > p - window) | (j < sinks))
    return seen


def attend(q, k, v, pos, scale, window=0, sinks=0):
    """One sequence: q [rows, Hq, d], k and v [keys, Hkv, d] (64 bits), pos [rows].  (o, lse, the same over |v|)."""
    rows, hq, d = q.shape
    G = hq // k.shape[1]
    o, lse, mag = torch.zeros_like(q, dtype=torch.float64), torch.zeros(rows, hq, dtype=torch.float64, device=q.device), None
    mag = torch.zeros_like(o)
    seen = visible(pos, k.shape[0], window, sinks)
    for h in range(hq):
        x = q[:, h].double() @ k[:, h // G].T * scale
        x = x.masked_fill(~seen, -math.inf)
        lse[:, h] = torch.logsumexp(x, 1)
        p = torch.exp(x - lse[:, h:h + 1])
        o[:, h], mag[:, h] = p @ v[:, h // G], p @ v[:, h // G].abs()
    return o, lse, mag


class Layout:
    """Sequences with segments [(start, length), ...] over a scattered block table."""

    def __init__(self, seqs, hq, hkv, d, seed=0, extra_blocks=3, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.seqs, self.hq, self.hkv, self.d, self.device = seqs, hq, hkv, d, device
        self.lens = [L for L, _ in seqs]
        counts = [-(-L // BS) for L in self.lens]
        self.max_blocks = max(counts + [1])
        self.num_blocks = sum(counts) + extra_blocks
        ids = torch.randperm(self.num_blocks, generator=g)
        table, n = torch.full((len(seqs), self.max_blocks), -1, dtype=torch.int32), 0
        for b, c in enumerate(counts):
            table[b, :c] = ids[n:n + c].to(torch.int32)
            n += c
        self.table = table.to(device)
        self.indptr = [0]
        for _, segs in seqs:
            self.indptr.append(self.indptr[-1] + len(segs))
        self.start = [a for _, segs in seqs for a, _ in segs]
        self.length = [n for _, segs in seqs for _, n in segs]
        self.pos_of = [[p for a, n in segs for p in range(a, a + n)] for _, segs in seqs]
        self.rows = sum(len(p) for p in self.pos_of)
        self.pos = torch.tensor([x for p in self.pos_of for x in p], dtype=torch.int64, device=device)
        self.seq = torch.tensor([b for b, p in enumerate(self.pos_of) for _ in p], dtype=torch.int64, device=device)

    def shape(self, msa, scale=None, **strides):
        return msa.make_shape(len(self.seqs), self.hq, self.hkv, self.d, self.max_blocks, self.num_blocks,
                              self.d ** -0.5 if scale is None else scale, **strides)

    def plan(self, msa, window=0, sinks=0, shape=None, **kw):
        args = (self.shape(msa) if shape is None else shape, self.lens, self.indptr, self.start, self.length)
        return msa.msa_plan_window(*args, window, sinks, **kw) if window else msa.msa_plan(*args, **kw)

    def places(self):
        """(block, token) of every packed row."""
        return self.table[self.seq, self.pos // BS].long(), self.pos % BS

    def keys(self, b, cache, is_v):
        """K or V [positions, heads, d] of sequence b from values [blocks, heads, 16, d] or [blocks, heads, d, 16]."""
        x = cache[self.table[b, :-(-self.lens[b] // BS)].long()]
        x = x.permute(0, 3, 1, 2) if is_v else x.permute(0, 2, 1, 3)
        return x.reshape(-1, self.hkv, self.d)[:self.lens[b]].double()

    def attend(self, q, k, v, window=0, sinks=0, scale=None):
        """(o, lse, o over |v|) of all rows; k and v the caches' values."""
        outs, row = [], 0
        for b, pos in enumerate(self.pos_of):
            n = len(pos)
            if n:
                outs.append(attend(q[row:row + n], self.keys(b, k, False), self.keys(b, v, True),
                                   self.pos[row:row + n], self.d ** -0.5 if scale is None else scale, window, sinks))
            row += n
        return [torch.cat(x) for x in zip(*outs)]


def normal(seed, *shape, device="cuda", dtype=torch.bfloat16):
    g = torch.Generator(device=device).manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device=device).normal_(generator=g)


def cache8(lay, seed):
    """A quantised cache of normal numbers: (K bytes, V bytes, K powers, V powers, K values, V values)."""
    dev = lay.device
    k = normal(seed, lay.num_blocks, lay.hkv, BS, lay.d, device=dev).double()
    v = normal(seed + 1, lay.num_blocks, lay.hkv, BS, lay.d, device=dev).double()
    k *= pow2(torch.randint(-4, 4, (lay.num_blocks, lay.hkv, BS, 1), generator=torch.Generator().manual_seed(seed)).to(dev)) ** 0.25
    v *= pow2(torch.randint(-8, 8, (lay.num_blocks, lay.hkv, BS, 1), generator=torch.Generator().manual_seed(seed + 1)).to(dev)) ** 0.25
    (kv, ks), (vv, vs) = quantise(k), quantise(v)
    kb = (kv / pow2(ks.long() - 127)[..., None]).float().to(torch.float8_e4m3fn).view(torch.uint8)
    vb = (vv / pow2(vs.long() - 127)[..., None]).float().to(torch.float8_e4m3fn).view(torch.uint8)
    return kb, vb.transpose(2, 3).contiguous(), ks, vs, kv, vv.transpose(2, 3).contiguous()


# Tolerances of attention outputs (o in bf16, lse in fp32).  A number rounded to bf16 is off by
# at most 2^-8 of itself: o once (2^-8 |o|), and the softmax weights p_j, but for those carried in two
# terms, each by up to 2^-8 p_j (together 2^-8 * sum_j p_j |v_j|; two terms: 2^-16).  Sums in 32
# bits over up to 10^4 keys add 10^4 * 2^-24 of that sum at most (6e-4; far less in practice), taken as 2^-12.
def o_bound(o, mag, precise=False):
    return 2.0 ** -8 * o.abs() + ((2.0 ** -16 if precise else 2.0 ** -8) + 2.0 ** -12) * mag + 1e-30


LSE = 2.5e-4
