"""Operators of encrypted decoder attention, measured against their plain forms.

What stands between the query/key/value projections and the attention products of a decoder, on ciphertexts: the position rotation
of queries and keys, the append of new tokens to a cache of pages, the masks of score rows, and the difference of two score maps.
A ciphertext holds, for token_inner tokens, the channels and heads of each token in its slots (the projections' token-shard
layout, features in channel-major order):
    slot = ((r * dim + d) * heads + h) * token_inner + t,     r < n / (dim * heads * token_inner) copies.
Score ciphertexts have the attention layout  slot = ((((e * P + pos) * heads + h) * token_inner + t) * R + r.

Ciphertexts and switching keys are uniform residues, which is what real ones look like; position tables and learned weights are
doubles.  Results on ciphertexts are residues, whole numbers that have to be equal: the order of every rounding is part of the
operators' definition.  The plain forms compute them with elementary torch operations, modular products of 50-bit words from a
double-precision quotient and wrapping 64-bit products.

Parameter sets (ring exponent: ciphertext primes, special primes, key-switch digits) are those of the other performance cases.
"""
import functools
import math

import numpy as np
import torch

own = False

PARAMS = {13: (6, 1, 6), 14: (6, 2, 3), 15: (12, 4, 3), 16: (24, 8, 3)}
SCALE = 2.0 ** 50


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the angles of one prompt of 128 tokens, 128 rotated channels per head: what a short call costs
        {"name": "table_128", "op": "table", "rot_dim": 128, "first": 0, "count": 128, "scaling": "none", "factor": 1.0},
        # a whole long context's table at once, wavelengths beyond the trained length stretched
        {"name": "table_long", "op": "table", "rot_dim": 128, "first": 0, "count": 131072, "scaling": "bands", "factor": 8.0},
        # one token of the toy ring (32 tokens x 64 features): launches and latency
        {"name": "rotary_toy", "op": "rotary", "log_n": 13, "level": 6, "dim": 16, "heads": 4, "inner": 32, "rot_dim": 16, "layout": "half",
         "shards": 1, "sets": 1, "same": True, "first": 77},
        # adjacent channels paired, three quarters of the head rotated: two rotations per ciphertext; a partial key-switch digit
        {"name": "rotary_part_interleaved", "op": "rotary", "log_n": 15, "level": 10, "dim": 64, "heads": 16, "inner": 16, "rot_dim": 48,
         "layout": "interleaved", "shards": 3, "sets": 2, "same": False, "first": 1000},
        # queries and keys of 128 tokens and 32 heads at the benchmark's parameters: a layer's prefill
        {"name": "rotary_128tokens", "op": "rotary", "log_n": 16, "level": 24, "dim": 128, "heads": 32, "inner": 8, "rot_dim": 128,
         "layout": "half", "shards": 16, "sets": 2, "same": False, "first": 0},
        # one generated token, its key rotated on the way, into one page
        {"name": "append_token", "op": "append", "log_n": 16, "level": 18, "dim": 128, "heads": 32, "inner": 8, "rot_dim": 128,
         "layout": "half", "items": 1, "ragged": True, "first": 1029},
        # three short sequences that end inside their pages
        {"name": "append_ragged", "op": "append", "log_n": 14, "level": 5, "dim": 32, "heads": 8, "inner": 16, "rot_dim": 20,
         "layout": "interleaved", "items": 3, "ragged": True, "first": 16},
        # the prompt of 125 tokens into sixteen pages, the last one not full
        {"name": "append_125tokens", "op": "append", "log_n": 16, "level": 18, "dim": 128, "heads": 32, "inner": 8, "rot_dim": 128,
         "layout": "half", "items": 16, "ragged": False, "first": 0},
        # causal rows of one score ciphertext of the toy ring
        {"name": "mask_toy", "op": "mask", "log_n": 13, "level": 5, "tokens": 16, "heads": 4, "block": 16, "inner": 4, "causal": True,
         "key_begin": 0, "key_end": 13, "window": 0, "offset": 0},
        # causal rows of 128 tokens and 32 heads, sixteen score ciphertexts after the exponential
        {"name": "mask_128tokens", "op": "mask", "log_n": 16, "level": 20, "tokens": 128, "heads": 32, "block": 8, "inner": 8,
         "causal": True, "key_begin": 0, "key_end": 125, "window": 0, "offset": 0},
        # the two maps of one group of the toy ring
        {"name": "difference_toy", "op": "difference", "log_n": 13, "level": 3, "tokens": 16, "heads": 4, "block": 16, "inner": 4},
        # the two maps of 128 tokens and 32 heads where the Softmax leaves them
        {"name": "difference_128tokens", "op": "difference", "log_n": 16, "level": 11, "tokens": 128, "heads": 32, "block": 8, "inner": 8},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["table", "rotary", "rotary", "rotary", "append", "append", "append", "mask", "mask", "difference", "difference"])
    if op == "table":
        return {"op": op, "rot_dim": 2 * rng.randint(2, 64), "first": rng.randint(0, 1 << 19), "count": _log_uniform(rng, 1, 100000),
                "scaling": rng.choice(["none", "linear", "base", "bands", "ramp"]), "factor": rng.choice([2.0, 4.0, 8.0, 32.0])}
    log_n = rng.choice([13, 14, 15, 16, 16])
    slots, L = 1 << (log_n - 1), PARAMS[log_n][0]
    if op in ("rotary", "append"):
        dim = rng.choice([16, 32, 64, 128])
        heads = rng.choice([h for h in (1, 2, 4, 8, 16, 32) if h * dim * 2 <= slots])
        room = slots // (dim * heads)
        inner = max(2, room // rng.choice([1, 1, 2]))
        case = {"op": op, "log_n": log_n, "level": rng.randint(2, L), "dim": dim, "heads": heads, "inner": inner,
                "rot_dim": rng.choice([dim, dim, 2 * rng.randint(1, dim // 2)]), "layout": rng.choice(["half", "interleaved"])}
        if op == "rotary":
            case |= {"shards": _log_uniform(rng, 1, 8), "sets": rng.choice([1, 2]), "same": rng.random() < 0.25, "first": rng.randint(0, 4000)}
        else:
            case |= {"items": _log_uniform(rng, 1, 12), "ragged": rng.random() < 0.6, "first": inner * rng.randint(0, 100) + rng.randint(0, inner - 1)}
        return case
    heads = rng.choice([1, 2, 4, 8, 16, 32])
    tokens = rng.choice([t for t in (2, 4, 8, 16, 32, 64, 128) if t * heads <= slots])
    block = rng.choice([b for b in (1, 2, 4, 8, 16, 32) if b <= tokens and b * tokens * heads <= slots and tokens // b <= 32])
    inner = rng.choice([t for t in (1, 2, 4, 8) if block % t == 0])
    case = {"op": op, "log_n": log_n, "level": rng.randint(2, L), "tokens": tokens, "heads": heads, "block": block, "inner": inner}
    if op == "mask":
        end = rng.randint(0, tokens)
        case |= {"causal": rng.random() < 0.6, "key_begin": rng.choice([0, 0, rng.randint(0, end)]), "key_end": end,
                 "window": rng.choice([0, 0, rng.randint(1, tokens)]), "offset": rng.choice([0, 0, rng.randint(0, tokens)])}
    return case


# ------------------------------------------------------------------------------------- a ring's plan for the plain forms
def _is_prime(n):
    d, s = n - 1, 0
    while d % 2 == 0:
        d, s = d // 2, s + 1
    for b in (2, 3, 5, 7, 11, 13, 17, 19, 23, 29, 31, 37):
        x = pow(b, d, n)
        if x in (1, n - 1):
            continue
        for _ in range(s - 1):
            x = x * x % n
            if x == n - 1:
                break
        else:
            return False
    return True


@functools.lru_cache(maxsize=None)
def _primes(log_n):
    """The largest primes below 2^50 that are 1 mod 2N: the special primes first, then the ciphertext primes.  (q..., p...)"""
    num_q, num_p, _ = PARAMS[log_n]
    m = 2 << log_n
    r, found = ((1 << 50) - 1) // m * m + 1, []
    while len(found) < num_q + num_p:
        if r < 1 << 50 and _is_prime(r):
            found.append(r)
        r -= m
    return found[num_p:] + found[:num_p]


def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _bitrev(x, bits):
    r = torch.zeros_like(x)
    for b in range(bits):
        r |= ((x >> b) & 1) << (bits - 1 - b)
    return r


def _mulmod(a, b, q):
    """a b mod q for 0 <= a, b < q < 2^50: the quotient from doubles is off by at most one, the remainder from wrapping products."""
    k = (a.double() * b.double() / q.double()).to(torch.int64)
    return torch.remainder(a * b - k * q, q)


class _Ring:
    """Tables of one parameter set: primes, powers of the roots, the slots' permutation, twiddles of the slots' transform."""

    def __init__(self, log_n):
        self.log_n, self.N, self.n = log_n, 1 << log_n, 1 << (log_n - 1)
        self.L, self.K, self.dnum = PARAMS[log_n]
        self.alpha = -(-self.L // self.dnum)
        self.primes = _primes(log_n)
        dev = self.dev = _device()
        N, n = self.N, self.n
        self.mod = torch.tensor(self.primes, dtype=torch.int64, device=dev)[:, None]         # [T][1]
        rev = _bitrev(torch.arange(N, device=dev), log_n)
        self.exponent = 2 * rev + 1                    # place p holds the value at psi^exponent[p]
        self.place = torch.empty(2 * N, dtype=torch.int64, device=dev)
        self.place[self.exponent] = torch.arange(N, device=dev)
        # psi: the smallest primitive 2N-th root of every prime
        some = []
        for q in self.primes:
            g = 2
            while pow(pow(g, (q - 1) // (2 * N), q), N, q) == 1:
                g += 1
            some.append(pow(g, (q - 1) // (2 * N), q))
        odd = self._powers(some)[:, 1::2]              # half of the primitive roots: the others are their negatives
        psi = [int(v) for v in torch.minimum(odd, self.mod - odd).min(dim=1).values]
        self.tw = self._powers(psi)[:, rev]                                                  # psi^bitrev(i)
        self.twi = self._powers([pow(r, -1, q) for r, q in zip(psi, self.primes)])[:, rev]
        # slots
        five, e = 1, []
        for _ in range(n):
            e.append((five - 1) // 4)
            five = five * 5 % (2 * N)
        self.slot_place = _bitrev(torch.tensor(e, device=dev), log_n - 1)                    # where slot j enters the transform
        t = range(n)
        f64 = functools.partial(torch.tensor, dtype=torch.float64, device=dev)
        self.omega = (f64([math.cos(2.0 * math.pi * k / n) for k in t]), f64([math.sin(2.0 * math.pi * k / n) for k in t]))
        self.zeta = (f64([math.cos(2.0 * math.pi * k / (2.0 * N)) for k in t]), f64([math.sin(2.0 * math.pi * k / (2.0 * N)) for k in t]))

    def _powers(self, roots):
        """[T][N] powers root^0 .. root^(N-1)."""
        w = torch.tensor(roots, dtype=torch.int64, device=self.dev)[:, None]
        p = torch.ones_like(w)
        while p.shape[1] < self.N:
            p = torch.cat([p, _mulmod(p, w, self.mod)], dim=1)
            w = _mulmod(w, w, self.mod)
        return p

    def limbs(self, level, special=False):
        """Prime indices of a polynomial: q_0 .. q_{level-1}, with the special primes behind them where asked for."""
        return list(range(level)) + (list(range(self.L, self.L + self.K)) if special else [])

    def galois(self, rotation):
        return pow(5, rotation % self.n, 2 * self.N)

    def sigma(self, g):
        """Places that the automorphism X -> X^g reads."""
        return self.place[(g * self.exponent) % (2 * self.N)]

    # transforms of [..., limbs, N]: coefficients in natural order, values in bit-reversed order
    def ntt(self, a, idx):
        shape, q, m = a.shape, self.mod[idx][:, :, None], 1
        while m < self.N:
            a = a.reshape(*shape[:-1], m, 2, self.N // (2 * m))
            u, v = a[..., 0, :], _mulmod(a[..., 1, :], self.tw[idx, m:2 * m][:, :, None], q)
            a = torch.stack([torch.remainder(u + v, q), torch.remainder(u - v, q)], dim=-2)
            m *= 2
        return a.reshape(shape)

    def intt(self, a, idx):
        shape, q, m = a.shape, self.mod[idx][:, :, None], self.N // 2
        while m >= 1:
            a = a.reshape(*shape[:-1], m, 2, self.N // (2 * m))
            u, v = a[..., 0, :], a[..., 1, :]
            a = torch.stack([torch.remainder(u + v, q), _mulmod(torch.remainder(u - v, q), self.twi[idx, m:2 * m][:, :, None], q)], dim=-2)
            m //= 2
        inv = torch.tensor([pow(self.N, -1, self.primes[i]) for i in idx], dtype=torch.int64, device=self.dev)[:, None]
        return _mulmod(a.reshape(shape), inv, self.mod[idx])

    def encode(self, z, scale, idx):
        """Slot values [..., n] to evaluations [..., limbs, N]: every product and every sum of the slots' transform is rounded on its own."""
        n = self.n
        re = torch.zeros_like(z)
        re[..., self.slot_place] = z
        im = torch.zeros_like(re)
        half = 1
        while half < n:
            wr, wi = self.omega[0][:: n // (2 * half)][:half], -self.omega[1][:: n // (2 * half)][:half]
            r, i = (x.reshape(*z.shape[:-1], n // (2 * half), 2, half) for x in (re, im))
            tr, ti = wr * r[..., 1, :] - wi * i[..., 1, :], wr * i[..., 1, :] + wi * r[..., 1, :]
            re = torch.stack([r[..., 0, :] + tr, r[..., 0, :] - tr], dim=-2).reshape(z.shape)
            im = torch.stack([i[..., 0, :] + ti, i[..., 0, :] - ti], dim=-2).reshape(z.shape)
            half *= 2
        wr, wi = self.zeta[0], -self.zeta[1]
        a, b, s = wr * re - wi * im, wr * im + wi * re, scale / n
        m = torch.cat([torch.round(a * s), torch.round(b * s)], dim=-1).to(torch.int64)
        return self.ntt(torch.remainder(m[..., None, :], self.mod[idx]), idx)

    # basis conversions (centred, of [..., sources, N] residues already multiplied by the inverse of their cofactor)
    def convert(self, y, src, dst):
        ps = [self.primes[i] for i in src]
        out = 0
        for a, i in enumerate(src):
            rest = math.prod(p for b, p in enumerate(ps) if b != a)
            w = torch.tensor([rest % self.primes[t] for t in dst], dtype=torch.int64, device=self.dev)[:, None]
            v = y[..., a, :]
            v = torch.where(v > self.primes[i] // 2, v - self.primes[i], v)[..., None, :]
            out = out + _mulmod(torch.remainder(v, self.mod[dst]), w, self.mod[dst])
        return torch.remainder(out, self.mod[dst])

    def cofactors(self, src):
        ps = [self.primes[i] for i in src]
        inv = [pow(math.prod(p for b, p in enumerate(ps) if b != a) % ps[a], -1, ps[a]) for a in range(len(ps))]
        return torch.tensor(inv, dtype=torch.int64, device=self.dev)[:, None]

    def modup(self, d, level):
        """The digits of [..., level, N] extended to all active primes: [..., digits, level + K, N], evaluation domain."""
        active, coef, digits = self.limbs(level, True), self.intt(d, self.limbs(level)), []
        for lo in range(0, level, self.alpha):
            src = list(range(lo, min(lo + self.alpha, level)))
            dst = [t for t in active if t not in src]
            y = _mulmod(coef[..., src, :], self.cofactors(src), self.mod[src])
            ext = self.ntt(self.convert(y, src, dst), dst)
            full = torch.empty(*d.shape[:-2], len(active), self.N, dtype=torch.int64, device=self.dev)
            full[..., [active.index(t) for t in dst], :] = ext
            full[..., src, :] = d[..., src, :]
            digits.append(full)
        return torch.stack(digits, dim=-3)

    def inner(self, ext, key, level):
        """<digits, key>: [..., 2, level + K, N]."""
        active = self.limbs(level, True)
        out = 0
        for j in range(ext.shape[-3]):
            out = out + _mulmod(ext[..., j, None, :, :], key[j][:, active], self.mod[active])
        return torch.remainder(out, self.mod[active])

    def moddown(self, u, level):
        """[..., level + K, N] divided by the product of the special primes."""
        special, idx = list(range(self.L, self.L + self.K)), self.limbs(level)
        y = _mulmod(self.intt(u[..., level:, :], special), self.cofactors(special), self.mod[special])
        conv = self.ntt(self.convert(y, special, idx), idx)
        P = math.prod(self.primes[i] for i in special)
        inv = torch.tensor([pow(P, -1, self.primes[i]) for i in idx], dtype=torch.int64, device=self.dev)[:, None]
        return _mulmod(torch.remainder(u[..., :level, :] - conv, self.mod[idx]), inv, self.mod[idx])

    def rescale(self, c):
        """[..., level, N] divided by the last prime."""
        last = c.shape[-2] - 1
        idx, q = self.limbs(last), self.primes[last]
        v = self.intt(c[..., last:, :], [last])
        lift = self.ntt(torch.remainder(torch.where(v > q // 2, v - q, v), self.mod[idx]), idx)
        inv = torch.tensor([pow(q, -1, self.primes[i]) for i in idx], dtype=torch.int64, device=self.dev)[:, None]
        return _mulmod(torch.remainder(c[..., :last, :] - lift, self.mod[idx]), inv, self.mod[idx])


@functools.lru_cache(maxsize=None)
def _ring(log_n):
    return _Ring(log_n)


@functools.lru_cache(maxsize=None)
def _context(log_n):
    """The framework's context of a parameter set: a program builds it once and keeps it."""
    from paper_2609_12378_b200 import binding
    num_q, _, dnum = PARAMS[log_n]
    primes = _primes(log_n)
    return binding.Context(log_n, primes[:num_q], primes[num_q:], dnum)


# -------------------------------------------------------------------------------------------------------------- prepare
THETA, ORIGINAL = 500000.0, 8192       # base of the angles, trained length


def _rotations(case):
    """Slot rotations that bring a channel its partner: one where the partner half a head away is reached both ways."""
    step = case["heads"] * case["inner"]
    apart = case["rot_dim"] // 2 if case["layout"] == "half" else 1
    return [apart * step] if 2 * apart == case["dim"] else [apart * step, -apart * step]


def _spans(case):
    """Per page of an append: first and last slot (of token_inner) that it fills, and the position of the first."""
    inner, spans = case["inner"], []
    for i in range(case["items"]):
        if case["ragged"]:        # sequences of their own, each at another place of its page
            begin = (case["first"] + 5 * i) % inner
            end = min(inner, begin + 1 + (7 * i) % inner)
            spans.append((begin, end, case["first"] + 3 * i))
        else:                     # one sequence, every page full but the last
            spans.append((0, inner if i + 1 < case["items"] else max(1, inner - 3), case["first"] + i * inner))
    return spans


class _Source:
    def __init__(self, log_n, seed):
        self.N, self.dev = 1 << log_n, _device()
        self.primes = _primes(log_n)
        self.num_q, _, self.dnum = PARAMS[log_n]
        self.gen = torch.Generator(device=self.dev)
        self.gen.manual_seed(seed)

    def residues(self, primes, *lead):
        out = torch.empty((*lead, len(primes), self.N), dtype=torch.int64, device=self.dev)
        for i, m in enumerate(primes):
            out[..., i, :] = torch.randint(0, m, (*lead, self.N), generator=self.gen, device=self.dev, dtype=torch.int64)
        return out

    def ciphertexts(self, count, level):
        return self.residues(self.primes[:level], count, 2)

    def keys(self, count):
        return self.residues(self.primes, count, self.dnum, 2)


def prepare(case, seed):
    s = {"case": case}
    if case["op"] == "table":
        s["first"] = case["first"] + seed % 1000          # every seed another stretch of the sequence
        return s
    src, level = _Source(case["log_n"], seed), case["level"]
    if case["op"] in ("rotary", "append"):
        inner = case["inner"]
        if case["op"] == "rotary":
            s["x"] = src.ciphertexts(case["shards"] * case["sets"], level)
            rows = case["shards"] if case["same"] else case["shards"] * inner
            s["rows"] = [i if case["same"] else i * inner for i in range(case["shards"])] * case["sets"]
        else:
            s["k"], s["v"] = src.ciphertexts(case["items"], level), src.ciphertexts(case["items"], level)
            s["spans"] = _spans(case)
            low = min(p for _, _, p in s["spans"])
            rows = max(p + e - b for b, e, p in s["spans"]) - low
            s["spans"] = [(b, e, p - low) for b, e, p in s["spans"]]
            # a pool of pages, of which the call names some in an order of its own
            s["page_k"], s["page_v"] = src.ciphertexts(case["items"] + 1, level - 1), src.ciphertexts(case["items"] + 1, level - 1)
            s["pages"] = [(3 * i + 1) % (case["items"] + 1) for i in range(case["items"])] if (case["items"] + 1) % 3 else list(range(case["items"], 0, -1))
        # the table of angles that the program keeps, from host arithmetic; a position of its own for every seed
        pos = np.arange(rows, dtype=np.float64)[:, None] + float(case["first"] + seed % 1000)
        angle = pos * THETA ** (-2.0 * np.arange(case["rot_dim"] // 2) / case["rot_dim"])
        s["cos"], s["sin"] = (torch.from_numpy(f(angle)).to(src.dev) for f in (np.cos, np.sin))
        s["rotations"] = _rotations(case)
        s["keys"] = src.keys(len(s["rotations"]))
    else:
        groups = case["tokens"] // case["block"]
        s["x"] = src.ciphertexts(groups, level)
        if case["op"] == "difference":
            s["y"] = src.ciphertexts(groups, level)
            s["weights"] = 0.2 + 0.6 * torch.rand(case["heads"], generator=src.gen, device=src.dev, dtype=torch.float64)
    _in_hand(s)
    return s


def _in_hand(s):
    """What a program holds beside the data: the plain forms' tables, or the framework's context, descriptors and output buffers."""
    case = s["case"]
    if not own:
        s["ring"] = _ring(case["log_n"])
        return
    from paper_2609_12378_b200 import binding
    ctx = s["ctx"] = _context(case["log_n"])

    def cts(t):
        return [binding.Ciphertext(x, SCALE) for x in t.view(torch.uint64)]

    def buffers(count, level):
        return torch.empty((count, 2, level, 1 << case["log_n"]), dtype=torch.int64, device=_device())

    for name in ("x", "y", "k", "v", "page_k", "page_v"):
        if name in s:
            s["ct_" + name] = cts(s[name])
    if "keys" in s:
        s["evk"] = [binding.SwitchKey(k, ctx.galois_element(r)) for k, r in zip(s["keys"].view(torch.uint64), s["rotations"])]
    if case["op"] == "append":
        s["out_k"], s["out_v"] = buffers(len(s["page_k"]), case["level"] - 1), buffers(len(s["page_v"]), case["level"] - 1)
        s["ct_out_k"], s["ct_out_v"] = cts(s["out_k"]), cts(s["out_v"])
        s["out_k"].copy_(s["page_k"]), s["out_v"].copy_(s["page_v"])
    else:
        s["out"] = buffers(len(s["x"]), case["level"] - 1)
        s["ct_out"] = cts(s["out"])


# ------------------------------------------------------------------------------------------------------------------ run
def _frequencies(case, pi=math.pi):
    """Angles per position of every rotated pair."""
    rot, f, kind = case["rot_dim"], case["factor"], case["scaling"]
    theta = THETA * f ** (rot / (rot - 2)) if kind == "base" else THETA
    out = []
    for j in range(rot // 2):
        w = theta ** (-2.0 * j / rot)
        if kind == "linear":
            w = w / f
        elif kind in ("bands", "ramp"):
            turns = ORIGINAL * w / (2.0 * pi)                 # turns within the trained length
            if kind == "bands":                               # up to 1 turn: stretched, from 4 on: kept, between: blended
                keep = min(1.0, max(0.0, (turns - 1.0) / (4.0 - 1.0)))
            else:                                             # blended along the pair's index, from 32 turns to 1
                at = [rot * math.log(ORIGINAL / (b * 2.0 * pi)) / (2.0 * math.log(theta)) for b in (32.0, 1.0)]
                lo, hi = max(0.0, math.floor(at[0])), min(rot - 1.0, math.ceil(at[1]))
                keep = 1.0 - min(1.0, max(0.0, (j - lo) / max(hi - lo, 0.001)))
            w = keep * w + (1.0 - keep) * (w / f)
        out.append(w)
    return out


def _magnitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "ramp" else 1.0


def _table(s):
    case = s["case"]
    w = torch.tensor(_frequencies(case), dtype=torch.float64, device=_device())
    pos = torch.arange(s["first"], s["first"] + case["count"], dtype=torch.float64, device=_device())
    angle = pos[:, None] * w
    return torch.cos(angle) * _magnitude(case), torch.sin(angle) * _magnitude(case)


def _position_slots(s, row, step, begin, end):
    """Slot vectors of one ciphertext: the factor of every channel, and of its partner for each rotation.  Token t of begin <= t < end
    takes row + (t - begin) step of the table; the other tokens get zeros."""
    case, R = s["case"], s["ring"]
    x = torch.arange(R.n, device=R.dev)
    t, d = x % case["inner"], x // (case["inner"] * case["heads"]) % case["dim"]
    rot, pairs = case["rot_dim"], case["rot_dim"] // 2
    j = d % pairs if case["layout"] == "half" else d // 2
    first = d < pairs if case["layout"] == "half" else d % 2 == 0
    rotated, live = d < rot, (t >= begin) & (t < end)
    at = (row + (t - begin) * step).clamp(0, len(s["cos"]) - 1), j.clamp(0, pairs - 1)
    cos, sin = s["cos"][at], s["sin"][at]
    zero = torch.zeros_like(cos)
    keep = torch.where(live, torch.where(rotated, cos, torch.ones_like(cos)), zero)
    sin = torch.where(live & rotated, sin, zero)
    if len(s["rotations"]) == 1:
        return [keep, torch.where(first, -sin, sin)]
    return [keep, torch.where(first, -sin, zero), torch.where(first, zero, sin)]


def _rotate_positions(s, c, slots):
    """rescale(C c + sum_r S_r rot_r(c)) with the products by S_r taken before the division by the special primes."""
    R, level = s["ring"], c.shape[-2]
    idx, wide = R.limbs(level), R.limbs(level, True)
    scale, q = float(R.primes[level - 1]), R.mod[R.limbs(level)]
    keep = R.encode(slots[0], scale, idx)
    out = _mulmod(c, keep, q)
    ext, total = R.modup(c[1], level), 0
    for r, rotation in enumerate(s["rotations"]):
        sigma = R.sigma(R.galois(rotation))
        pt = R.encode(slots[1 + r], scale, wide)
        total = total + _mulmod(R.inner(ext[..., sigma], s["keys"][r], level), pt, R.mod[wide])
        out[0] = torch.remainder(out[0] + _mulmod(c[0][..., sigma], pt[:level], q), q)
    down = R.moddown(torch.remainder(total, R.mod[wide]), level)
    return R.rescale(torch.remainder(out + down, q))


def _rotary(s):
    case = s["case"]
    step = 0 if case["same"] else 1
    return torch.stack([_rotate_positions(s, c, _position_slots(s, row, step, 0, case["inner"])) for c, row in zip(s["x"], s["rows"])])


def _append(s):
    R, level = s["ring"], s["case"]["level"]
    idx = R.limbs(level - 1)
    out_k, out_v = s["page_k"].clone(), s["page_v"].clone()
    for i, (page, (begin, end, row)) in enumerate(zip(s["pages"], s["spans"])):
        slots = _position_slots(s, row, 1, begin, end)
        out_k[page] = torch.remainder(out_k[page] + _rotate_positions(s, s["k"][i], slots), R.mod[idx])
        if end - begin == s["case"]["inner"]:                  # a full page takes the values as they are
            v = s["v"][i][:, :level - 1]
        else:
            t = torch.arange(R.n, device=R.dev) % s["case"]["inner"]
            live = ((t >= begin) & (t < end)).double()
            v = R.rescale(_mulmod(s["v"][i], R.encode(live, float(R.primes[level - 1]), R.limbs(level)), R.mod[R.limbs(level)]))
        out_v[page] = torch.remainder(out_v[page] + v, R.mod[idx])
    return [out_k, out_v]


def _score_places(s):
    """(block, query token, head) of every slot of a score ciphertext."""
    case, R = s["case"], s["ring"]
    copies = R.n // (case["block"] * case["tokens"] * case["heads"])
    x = torch.arange(R.n, device=R.dev) // copies
    t, h = x % case["inner"], x // case["inner"] % case["heads"]
    pos = x // (case["inner"] * case["heads"])
    per = case["tokens"] // case["inner"]
    return pos // per, pos % per * case["inner"] + t, h


def _mask(s):
    case, R, x = s["case"], s["ring"], s["x"]
    level, T, E = case["level"], case["tokens"], case["block"]
    e, i, _ = _score_places(s)
    q, out = R.mod[R.limbs(level)], []
    for g in range(T // E):
        f = i + g * E                                          # the key operand, rotated by g blocks of tokens over (block, token)
        key = torch.where(f < T, (f + e) % T, (f - T + (e + 1) % E) % T)
        at = i + case["offset"]
        live = (key >= case["key_begin"]) & (key < case["key_end"])
        if case["causal"]:
            live &= key <= at
        if case["window"]:
            live &= key + case["window"] > at
        out.append(R.rescale(_mulmod(x[g], R.encode(live.double(), float(R.primes[level - 1]), R.limbs(level)), q)))
    return torch.stack(out)


def _difference(s):
    R, level = s["ring"], s["case"]["level"]
    _, _, h = _score_places(s)
    q = R.mod[R.limbs(level)]
    pt = R.encode(s["weights"][h], float(R.primes[level - 1]), R.limbs(level))
    return torch.stack([torch.remainder(x[:, :level - 1] - R.rescale(_mulmod(y, pt, q)), q[:level - 1]) for x, y in zip(s["x"], s["y"])])


_PLAIN = {"table": _table, "rotary": _rotary, "append": _append, "mask": _mask, "difference": _difference}


def run(s):
    case = s["case"]
    if not own:
        return _PLAIN[case["op"]](s)
    if case["op"] == "table":
        # a program's context for the positions alone: any parameter set serves
        return _context(13).rotary_table(case["rot_dim"], s["first"], case["count"], theta=THETA, scaling=case["scaling"], factor=case["factor"],
                                         original_length=ORIGINAL, magnitude=_magnitude(case))
    ctx = s["ctx"]
    if case["op"] == "rotary":
        ctx.rotary(s["ct_x"], s["rows"], s["cos"], s["sin"], s["evk"], case["dim"], case["heads"], case["inner"], rot_dim=case["rot_dim"],
                   layout=case["layout"], same_position=case["same"], outs=s["ct_out"])
        return s["out"]
    if case["op"] == "append":
        ctx.cache_append(s["ct_k"], s["ct_v"], s["pages"], s["spans"], s["ct_page_k"], s["ct_page_v"], s["cos"], s["sin"], s["evk"], case["dim"],
                         case["heads"], case["inner"], rot_dim=case["rot_dim"], layout=case["layout"], out_k=s["ct_out_k"], out_v=s["ct_out_v"])
        return [s["out_k"], s["out_v"]]
    if case["op"] == "mask":
        ctx.attention_mask(s["ct_x"], case["tokens"], case["heads"], case["block"], token_inner=case["inner"], causal=case["causal"],
                           key_begin=case["key_begin"], key_end=case["key_end"], window=case["window"], query_offset=case["offset"], outs=s["ct_out"])
        return s["out"]
    ctx.attention_difference(s["ct_x"], s["ct_y"], s["weights"], case["tokens"], case["heads"], case["block"], token_inner=case["inner"], outs=s["ct_out"])
    return s["out"]


# ---------------------------------------------------------------------------------------------------------------- exact
def exact(case, seed):
    """Angles in extended precision.  Residues have no value beside the one that the definition's order of roundings gives them."""
    if case["op"] != "table" or case["count"] * case["rot_dim"] > 1 << 25:
        return None
    ld = np.longdouble
    rot, j = ld(case["rot_dim"]), np.arange(case["rot_dim"] // 2, dtype=np.longdouble)
    pi = ld("3.14159265358979323846264338327950288")
    theta, f, kind = ld(THETA), ld(case["factor"]), case["scaling"]
    if kind == "base":
        theta = theta * f ** (rot / (rot - 2))
    w = theta ** (-2 * j / rot)
    if kind == "linear":
        w = w / f
    elif kind == "bands":
        keep = np.clip((ORIGINAL * w / (2 * pi) - 1) / 3, 0, 1)
        w = w * (keep + (1 - keep) / f)
    elif kind == "ramp":
        edge = [rot * np.log(ORIGINAL / (ld(b) * 2 * pi)) / (2 * np.log(theta)) for b in (32, 1)]
        lo, hi = max(ld(0), np.floor(edge[0])), min(rot - 1, np.ceil(edge[1]))
        keep = 1 - np.clip((j - lo) / max(hi - lo, ld("0.001")), 0, 1)
        w = w * (keep + (1 - keep) / f)
    m = ld("0.1") * np.log(f) + 1 if kind == "ramp" else ld(1)
    pos = np.arange(case["count"], dtype=np.longdouble) + (case["first"] + seed % 1000)
    angle = np.remainder(pos[:, None] * w, 2 * pi)
    return [(np.cos(angle) * m).astype(np.float64), (np.sin(angle) * m).astype(np.float64)]


# ----------------------------------------------------------------------------------------------------------------- work
def work(case):
    """Bytes: ciphertexts, keys, pages and tables once.  Operations: six double-precision operations for a modular product of 50-bit
    words, two more for a butterfly, one more where a product is added to a sum."""
    if case["op"] == "table":
        values = case["count"] * case["rot_dim"]
        return {"bytes": 8.0 * values, "flops": 20.0 * values}
    log_n, level = case["log_n"], case["level"]
    N, (L, K, dnum) = 1 << log_n, PARAMS[case["log_n"]]
    alpha, limb, pair, ntt = -(-L // dnum), 8 * N, 7 * N, 8 * (N // 2) * log_n
    ct = lambda l: 2 * l * limb  # noqa: E731
    encode = lambda limbs: 5 * (N // 2) * (log_n - 1) + limbs * ntt  # noqa: E731
    rescale = 2 * level * ntt + 2 * (level - 1) * pair
    digits = [min(alpha, level - lo) for lo in range(0, level, alpha)]
    nt = level + K

    def positions(count, distinct):
        rotations = len(_rotations(case))
        flops = count * ((level + sum(nt - d for d in digits)) * ntt + pair * sum(d * (nt - d) for d in digits))       # extension
        flops += count * rotations * (len(digits) + 1) * 2 * nt * pair                                                  # keys, factors
        flops += count * (2 * K * ntt + 2 * level * (K + 1) * pair + 2 * level * pair) + count * rescale               # division, own factor
        flops += distinct * (encode(level) + rotations * encode(nt))
        return rotations * len(digits) * 2 * nt * limb, flops

    if case["op"] == "rotary":
        count = case["shards"] * case["sets"]
        keys, flops = positions(count, case["shards"])
        rows = case["shards"] * (1 if case["same"] else case["inner"])
        return {"bytes": keys + count * (ct(level) + ct(level - 1)) + 8.0 * rows * case["rot_dim"], "flops": float(flops)}
    if case["op"] == "append":
        spans = _spans(case)
        keys, flops = positions(len(spans), len(spans))
        whole = sum(e - b == case["inner"] for b, e, _ in spans)
        part = len(spans) - whole
        flops += part * (encode(level) + 2 * level * pair + rescale)
        moved = len(spans) * (ct(level) + 4 * ct(level - 1)) + part * ct(level) + whole * ct(level - 1)
        return {"bytes": keys + moved + 8.0 * sum(e - b for b, e, _ in spans) * case["rot_dim"], "flops": float(flops)}
    groups = case["tokens"] // case["block"]
    flops = groups * (2 * level * pair + rescale)
    if case["op"] == "mask":
        return {"bytes": float(groups * (ct(level) + ct(level - 1))), "flops": float(flops + groups * encode(level))}
    return {"bytes": float(groups * (ct(level) + 2 * ct(level - 1))), "flops": float(flops + encode(level))}
