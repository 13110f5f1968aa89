"""The 8-bit cache operators as measurable cases: writing rows into a quantised cache (a whole
compressed prompt, a chunk, one token), reading rows back, and decode attention over it.

A pass is one call of `paper_2607_16213_gb300.api` on device tensors (`quant_append`, `quant_read`,
`decode_quant`), with the cache and the workspace kept across calls as a serving program keeps
them.  A pass that appends first puts the lengths back to where the case starts, as a program does
that tries another continuation of the same prompt; the rows written before are written over.

The cache: codes [B][Hkv][m_cap][d] in 8 bits and a scale per `block` rows and head.  A block whose
first row is written by a call gets the smallest scale s with s * qmax >= the largest finite magnitude
of its rows, among the powers of two (e4m3, qmax 448) or the numbers of 4 significant bits
(int8, qmax 127), at least 2^-100.  A block that holds rows already doubles its scale as often as the new
rows need and encodes the old codes anew.  Codes round x / s to nearest even.

Inputs: rows of segments around a random centroid, 1% of the positions four times larger, 3% of
the key channels eight times larger, drawn on the device from the seed.
"""
import math

import torch

own = False

_LLAMA = dict(dtype="bf16", hq=32, hkv=8, d=128)
_SMALL = dict(dtype="fp32", hq=4, hkv=2, d=64)
_QMAX = {"e4m3": 448.0, "int8": 127.0}
_MIN_SCALE = 2.0 ** -100


def listed():
    def append(name, batch, start, rows, cache, block, shape=_LLAMA, ragged=False):
        return dict(name=name, kind="append", batch=batch, start=start, rows=rows, cache=cache, block=block, ragged=ragged, **shape)

    def read(name, batch, rows, cache, block, shape=_LLAMA, ragged=False):
        return dict(name=name, kind="read", batch=batch, start=rows, rows=rows, cache=cache, block=block, ragged=ragged, **shape)

    def decode(name, batch, rows, cache, block, shape=_LLAMA, ragged=False, bias=True, new=True):
        return dict(name=name, kind="decode", batch=batch, start=rows, rows=1, cache=cache, block=block, ragged=ragged, bias=bias,
                    new=new, **shape)

    return [
        # a chunk of a small fp32 model behind an odd number of rows: latency
        append("append_fp32_37", 2, 201, 37, "int8", 32, _SMALL),
        # the compressed cache of a 100k prompt, one layer, into an empty 8-bit cache
        append("append_25k", 1, 0, 25000, "e4m3", 64),
        # a serving batch of ragged compressed prompts
        append("append_b64_2k", 64, 0, 2048, "int8", 32, ragged=True),
        # the uncompressed cache of a long prompt, the largest case
        append("append_131k", 1, 0, 131072, "e4m3", 128),
        # a small fp32 cache read back for a check or a hand-over
        read("read_fp32_1k", 1, 1000, "int8", 16, _SMALL),
        # eight ragged caches read back, to be compressed again
        read("read_b8_16k", 8, 16384, "e4m3", 64, ragged=True),
        # a token of a small fp32 model
        decode("decode_fp32_256", 1, 256, "int8", 16, _SMALL),
        # a token of the long-context setting (a 100k prompt at 25%)
        decode("decode_25k", 1, 25000, "e4m3", 64),
        # a token of a large ragged batch over short caches
        decode("decode_b64_819", 64, 819, "int8", 32, ragged=True),
        # a token of eight ragged long caches
        decode("decode_b8_16k", 8, 16384, "e4m3", 128, ragged=True),
        # a wide query group over narrow heads, many tokens' caches of a ragged batch
        decode("decode_g8_d64", 16, 5000, "int8", 64, dict(_LLAMA, hq=64, d=64), ragged=True),
        # a token over an uncompressed cache: no bias, nothing appended
        decode("decode_131k_plain", 1, 131072, "e4m3", 64, bias=False, new=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: batches of up to 64, caches of 40 to 131072 rows (at most 1M rows of
    all sequences and heads), every block size, both codes and types."""
    kind = rng.choice(("append", "read", "decode", "decode"))
    fp32 = rng.random() < 0.25
    hq, hkv = rng.choice(((32, 8), (32, 8), (64, 8), (32, 32), (32, 4), (32, 2)))
    if fp32 and rng.random() < 0.7:
        hq, hkv = 4, 2
    d = rng.choice((128, 128, 64))
    batch = rng.choice((1, 1, 2, 5, 8, 16, 33, 64))
    most = (400000 if fp32 else 1000000) // (batch * hkv)
    case = dict(kind=kind, batch=batch, cache=rng.choice(("e4m3", "int8")), block=rng.choice((16, 32, 64, 128)),
                ragged=batch > 1 and rng.random() < 0.8, dtype="fp32" if fp32 else "bf16", hq=hq, hkv=hkv, d=d)
    rows = _log_int(rng, 40, max(41, min(131072, most)))
    if kind == "append":
        if rng.random() < 0.4:  # a chunk behind what is there
            chunk = _log_int(rng, 1, max(2, min(4096, rows)))
            return dict(case, start=max(1, rows - chunk), rows=chunk)
        return dict(case, start=0, rows=rows)
    if kind == "read":
        return dict(case, start=rows, rows=rows)
    return dict(case, start=rows, rows=1, bias=rng.random() < 0.8, new=rng.random() < 0.8)


# ---- inputs ----------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _code_dtype(case):
    return torch.float8_e4m3fn if case["cache"] == "e4m3" else torch.int8


def _ragged(case, n):
    """Per sequence all n rows, or from about half of them up; of the case's sizes alone."""
    if not case["ragged"] or n < 2:
        return [n] * case["batch"]
    lo = (n + 1) // 2
    return [lo + ((i * 2654435761 + 12345) % 1000003) * (n - lo + 1) // 1000003 for i in range(case["batch"])]


def _rows(g, B, H, n, d, dtype, keys):
    """Rows [B][H][n][d] in segments of 16 around random centroids."""
    out = torch.empty((B, H, n, d), dtype=dtype, device="cuda")
    large = 1.0 + 3.0 * (torch.rand((B, 1, n, 1), generator=g, device="cuda") < 0.01).float()
    loud = 1.0 + 7.0 * (torch.rand((H, 1, d), generator=g, device="cuda") < 0.03).float()
    for b in range(B):
        cent = torch.randn((H, (n + 15) // 16, d), generator=g, device="cuda")
        x = torch.randn((H, n, d), generator=g, device="cuda").mul_(0.4).add_(cent.repeat_interleave(16, 1)[:, :n])
        out[b] = (x.mul_(large[b]).mul_(loud) if keys else x).to(dtype)
    return out


def _bias(g, B, H, n):
    """What a compression leaves: alpha ln R >= 0, the same for every KV head, about one in eight positive."""
    merged = torch.rand((B, 1, n), generator=g, device="cuda") < 0.125
    ratio = 1.0 + torch.empty((B, 1, n), device="cuda").exponential_(0.25, generator=g) * merged
    return (0.5 * torch.log(ratio)).expand(B, H, n).contiguous()


class _State:
    """A cache with `start` rows, and what one pass takes."""

    def __init__(self, case, seed):
        self.case = case
        g = torch.Generator(device="cuda")
        g.manual_seed(int(seed))
        B, H, d, n = case["batch"], case["hkv"], case["d"], case["rows"]
        decode = case["kind"] == "decode"
        self.block = case["block"]
        most = case["start"] + (n if case["kind"] == "append" else 0)
        self.cap = (most + (1 if decode else 0) + 63) // 64 * 64
        blocks = -(-self.cap // self.block)
        self.K, self.V = (torch.zeros((B, H, self.cap, d), dtype=torch.int8, device="cuda").view(_code_dtype(case)) for _ in range(2))
        self.K_scale, self.V_scale = (torch.zeros((B, H, blocks), device="cuda") for _ in range(2))
        self.bias = torch.zeros((B, H, self.cap), device="cuda") if case.get("bias", True) else None
        self.lengths = torch.zeros((B,), dtype=torch.int32, device="cuda")
        if case["start"]:
            starts = _ragged(case, case["start"])
            counts = torch.tensor(starts, dtype=torch.int32, device="cuda")
            _append(self, _rows(g, B, H, case["start"], d, _dtype(case), True), _rows(g, B, H, case["start"], d, _dtype(case), False),
                    _bias(g, B, H, case["start"]), counts)
        self.base = self.lengths.clone()
        if case["kind"] == "append":
            self.k, self.v = _rows(g, B, H, n, d, _dtype(case), True), _rows(g, B, H, n, d, _dtype(case), False)
            self.b = _bias(g, B, H, n)
            self.counts = torch.tensor(_ragged(case, n), dtype=torch.int32, device="cuda")
        elif case["kind"] == "read":
            self.k_out, self.v_out = (torch.zeros((B, H, n, d), dtype=_dtype(case), device="cuda") for _ in range(2))
        else:
            self.q = torch.randn((B, case["hq"], d), generator=g, device="cuda").to(_dtype(case))
            self.k = self.v = None
            if case["new"]:
                self.k, self.v = (torch.randn((B, H, d), generator=g, device="cuda").to(_dtype(case)) for _ in range(2))
            self.out = torch.zeros_like(self.q)
        self.handle = None


def prepare(case, seed):
    return _State(case, seed)


# ---- the plain form --------------------------------------------------------------------------
def _two(e):
    """2^e in 32 bits, exactly, from its bits (a power may be a last place off); -126 <= e <= 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _fresh_scale(amax, cache):
    """The smallest scale of the grid with scale * qmax >= amax (in 64 bits: amax may lie on the border)."""
    # (by a tensor: a division by a number may become a product with its rounded inverse)
    m, e = torch.frexp((amax.double() / torch.full_like(amax, _QMAX[cache], dtype=torch.float64)).clamp_min(_MIN_SCALE))
    m = torch.where(m > 0.5, 1.0, 0.5) if cache == "e4m3" else torch.ceil(m * 16) / 16
    return m.float() * _two(e)


def _grown_scale(amax, old, cache):
    """old * 2^k with the smallest k >= 0 that covers amax."""
    old = old.clamp_min(_MIN_SCALE)
    most = old * _QMAX[cache]
    k = (torch.frexp(amax).exponent - torch.frexp(most).exponent).clamp_min(0)
    k = torch.where(amax > most, k + (most * _two(k.clamp_max(126)) < amax), 0)
    return old * _two(k.clamp_max(126))


def _encode(x, cache):
    """Codes of x / scale, as bytes (in 64 bits: quotients may lie next to the border of two codes)."""
    x = x.clamp(-_QMAX[cache], _QMAX[cache])
    if cache == "e4m3":
        return x.float().to(torch.float8_e4m3fn).view(torch.int8)
    return torch.round(x).nan_to_num(0.0).to(torch.int8)


def _values(codes):
    return codes.float()


def _store(codes, scale, x, lengths, n, block, cache):
    """Rows t < n[b] of x [B][H][T][d] to row lengths[b] + t of the codes (in place)."""
    B, H, T, d = x.shape
    cap, blocks = codes.shape[2], scale.shape[2]
    raw = codes.view(torch.int8)
    t = torch.arange(T, device="cuda")
    pos = lengths[:, None].long() + t
    valid = t < n[:, None]
    blk = torch.where(valid, pos // block, blocks)
    a = x.float().abs().nan_to_num(0.0, 0.0, 0.0).amax(3)
    amax = torch.zeros((B, H, blocks + 1), device="cuda").scatter_reduce_(2, blk[:, None].expand(B, H, T), a, "amax")[:, :, :blocks]
    touched = torch.zeros((B, blocks + 1), dtype=torch.bool, device="cuda").scatter_(1, blk, True)[:, None, :blocks]
    part = (lengths.long() // block)[:, None, None]
    holds = (torch.arange(blocks, device="cuda") == part) & (lengths % block != 0)[:, None, None]
    fresh, grown = _fresh_scale(amax, cache), _grown_scale(amax, scale, cache)
    new = torch.where(touched, torch.where(holds, grown, fresh), scale)
    # the rows that the partly filled block holds, under its new scale
    at = part * block + torch.arange(block, device="cuda")
    old = at < lengths[:, None, None]
    at = at.clamp_max(cap - 1).expand(B, H, block)
    ratio = torch.where(touched & holds, scale.clamp_min(_MIN_SCALE) / new, 1.0).gather(2, part.clamp_max(blocks - 1).expand(B, H, 1))
    idx = at[..., None].expand(B, H, block, d)
    rows = codes.view(torch.int8).gather(2, idx)
    again = _encode(_values(rows.view(codes.dtype)).double() * ratio[..., None], cache)
    grew = (ratio != 1.0)[..., None] & old[..., None]
    rows = torch.where(grew, again, rows)
    b4 = torch.arange(B, device="cuda")[:, None, None]
    h4 = torch.arange(H, device="cuda")[None, :, None]
    keep = grew.expand(B, H, block, 1)[..., 0]
    raw[b4.expand_as(at)[keep], h4.expand_as(at)[keep], at[keep]] = rows[keep]
    s = new.gather(2, blk.clamp_max(blocks - 1)[:, None].expand(B, H, T))
    put = valid[:, None].expand(B, H, T)
    step = max(1, (1 << 27) // max(1, T * d))
    y = torch.cat([_encode(x.reshape(B * H, T, d)[i:i + step].double() / s.reshape(B * H, T, 1)[i:i + step], cache)
                   for i in range(0, B * H, step)]).view(B, H, T, d)
    p3 = pos[:, None].expand(B, H, T)
    raw[b4.expand_as(p3)[put], h4.expand_as(p3)[put], p3[put]] = y[put]
    scale.copy_(new)


def _append(st, k, v, bias, counts):
    block, cache = st.block, st.case["cache"]
    n = torch.minimum(counts, st.cap - st.lengths)
    _store(st.K, st.K_scale, k, st.lengths, n, block, cache)
    _store(st.V, st.V_scale, v, st.lengths, n, block, cache)
    if st.bias is not None:
        T = k.shape[2]
        pos = st.lengths[:, None].long() + torch.arange(T, device="cuda")
        put = (torch.arange(T, device="cuda") < n[:, None])[:, None].expand(-1, k.shape[1], -1)
        b, h = torch.meshgrid(torch.arange(k.shape[0], device="cuda"), torch.arange(k.shape[1], device="cuda"), indexing="ij")
        p3 = pos[:, None].expand_as(put)
        st.bias[b[..., None].expand_as(p3)[put], h[..., None].expand_as(p3)[put], p3[put]] = bias[put] if bias is not None else 0.0
    st.lengths += n


def _dequantised(codes, scale, block):
    return _values(codes) * scale.repeat_interleave(block, 2)[:, :, :codes.shape[2], None]


def _read(st):
    """Rows below the lengths; the others of the output stay."""
    n = st.k_out.shape[2]
    live = (torch.arange(n, device="cuda") < st.lengths[:, None])[:, None, :, None]
    for codes, scale, out in ((st.K, st.K_scale, st.k_out), (st.V, st.V_scale, st.v_out)):
        out.copy_(torch.where(live, _dequantised(codes[:, :, :n], scale, st.block).to(out.dtype), out))


def _decode(st):
    B, Hq, d = st.q.shape
    H = st.K.shape[1]
    q = st.q.float().view(B, H, Hq // H, d) / math.sqrt(d)
    K, V = _dequantised(st.K, st.K_scale, st.block), _dequantised(st.V, st.V_scale, st.block)
    s = q @ K.transpose(2, 3)
    if st.bias is not None:
        s = s + st.bias[:, :, None]
    s = s.masked_fill((torch.arange(st.cap, device="cuda") >= st.lengths[:, None])[:, None, None], -math.inf)
    V = V.masked_fill((torch.arange(st.cap, device="cuda") >= st.lengths[:, None])[:, None, :, None], 0.0)
    if st.k is not None:
        s = torch.cat([s, q @ st.k.float()[..., None]], 3)
        V = torch.cat([V, st.v.float()[:, :, None]], 2)
    m = s.amax(3, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    z = p.sum(3, keepdim=True)
    st.out.copy_((p @ V / torch.where(z > 0, z, 1.0)).view(B, Hq, d))
    if st.k is not None:
        _append(st, st.k[:, :, None], st.v[:, :, None], None, torch.ones_like(st.lengths))


# ---- one pass --------------------------------------------------------------------------------
def _handle(st):
    """The framework's cache over the state's tensors, and a workspace."""
    import paper_2607_16213_gb300 as S
    from paper_2607_16213_gb300 import api
    c = st.case
    shape = api.make_shape(c["dtype"], c["batch"], c["hq"], c["hkv"], c["d"], 32, st.cap, st.cap)
    cache = api.QuantCache(shape, c["cache"], st.block, st.K, st.V, st.K_scale, st.V_scale, st.bias, st.lengths)
    size = S.selkv_decode_q_workspace_size if c["kind"] == "decode" else S.selkv_qcache_workspace_size
    return api, cache, api.Workspace(size(shape))


def run(st):
    kind = st.case["kind"]
    appends = kind == "append" or (kind == "decode" and st.k is not None)
    if appends:
        st.lengths.copy_(st.base)
    if own:
        if st.handle is None:
            st.handle = _handle(st)
        api, cache, ws = st.handle
        if kind == "append":
            api.quant_append(cache, st.k, st.v, st.b, st.counts, workspace=ws)
        elif kind == "read":
            api.quant_read(cache, out=(st.k_out, st.v_out), workspace=ws)
        else:
            api.decode_quant(cache, st.q, st.k, st.v, out=st.out, workspace=ws)
    elif kind == "append":
        _append(st, st.k, st.v, st.b, st.counts)
    elif kind == "read":
        _read(st)
    else:
        _decode(st)
    if kind == "read":
        return dict(K=st.k_out, V=st.v_out)
    got = dict(out=st.out) if kind == "decode" else {}
    if appends:
        got.update(K=st.K, V=st.V, K_scale=st.K_scale, V_scale=st.V_scale, lengths=st.lengths)
        if st.bias is not None:
            got["bias"] = st.bias
    return got


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    B, Hq, H, d, block = case["batch"], case["hq"], case["hkv"], case["d"], case["block"]
    rows = sum(_ragged(case, case["rows"] if case["kind"] == "append" else case["start"]))
    scales = 2 * 4 * H * -(-rows // block)
    if case["kind"] == "append":
        # rows and bias in, codes, scales and bias out; largest magnitude, quotient and rounding of each value
        return dict(bytes=2 * H * rows * d * (e + 1) + 8 * H * rows + scales, flops=6.0 * H * rows * d)
    if case["kind"] == "read":
        return dict(bytes=2 * H * rows * d * (e + 1) + scales, flops=2.0 * H * rows * d)
    # the cache and one bias row for all heads; queries and output; the new row in and out
    by = 2 * H * rows * d + scales + (4 * rows if case["bias"] else 0) + 2 * B * Hq * d * e
    if case["new"]:
        by += 2 * B * H * d * (e + 1)
    return dict(bytes=by, flops=4.0 * Hq * d * rows)


# ---- the same in 64 bits ---------------------------------------------------------------------
def _exact_value(byte, cache):
    """What codes stand for, from their bits."""
    if cache == "int8":
        return byte.double()
    u = byte.view(torch.uint8).int()
    e, m, sign = (u >> 3) & 15, (u & 7).double(), 1.0 - 2.0 * (u >> 7).double()
    v = torch.where(e > 0, (8.0 + m) * _exact_two(e - 10), m * 2.0 ** -9)
    return sign * torch.where((u & 127) == 127, math.nan, v)


def _exact_two(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_round(y, cache):
    """y to the nearest value of a code, ties to even."""
    if cache == "int8":
        return torch.round(y)
    step = _exact_two(torch.frexp(y.abs().clamp_min(2.0 ** -6)).exponent - 4)
    return torch.round(y / step) * step


def _exact_store(value, scale, x, L, block, cache):
    """value [H][cap][d] (what the codes stand for, without their scale) and scale [H][blocks] with the
    rows x [H][n][d] behind the first L, block by block."""
    n = x.shape[1]
    for p in range(L // block, -(-(L + n) // block)):
        r0, r1 = max(L, p * block), min(L + n, (p + 1) * block)
        xb = x[:, r0 - L:r1 - L].double()
        most = xb.abs().amax((1, 2))
        need = most / torch.full_like(most, _QMAX[cache])
        if r0 > p * block:  # rows are there
            s0 = scale[:, p].double()
            m, e = torch.frexp(need / s0)
            s = s0 * _exact_two((e - (m == 0.5).int()).clamp_min(0))
            value[:, p * block:r0] = _exact_round(value[:, p * block:r0] * (s0 / s)[:, None, None], cache)
        else:
            two = _exact_two(torch.frexp(need).exponent - 1)  # two <= need < 2 two
            s = two * torch.ceil(need / two) if cache == "e4m3" else two * torch.ceil(8.0 * (need / two)) / 8.0
        scale[:, p] = s
        value[:, r0:r1] = _exact_round(xb / s[:, None, None], cache)


def exact(case, seed):
    st = _State(case, seed)
    cache, block, H = case["cache"], case["block"], case["hkv"]
    lens = st.base.tolist()
    if case["kind"] == "read":
        outs = []
        for codes, scale in ((st.K, st.K_scale), (st.V, st.V_scale)):
            o = torch.zeros(st.k_out.shape, dtype=torch.float64, device="cuda")
            for b, n in enumerate(lens):
                at = torch.arange(n, device="cuda") // block
                o[b, :, :n] = _exact_value(codes[b, :, :n].view(torch.int8), cache) * scale[b].double()[:, at, None]
            outs.append(o)
        return dict(K=outs[0], V=outs[1])
    got = {}
    if case["kind"] == "decode":
        got["out"] = torch.zeros(st.q.shape, dtype=torch.float64, device="cuda")
        G = case["hq"] // H
        for b, n in enumerate(lens):
            at = torch.arange(n, device="cuda") // block
            for h in range(H):
                k = _exact_value(st.K[b, h, :n].view(torch.int8), cache) * st.K_scale[b, h].double()[at, None]
                v = _exact_value(st.V[b, h, :n].view(torch.int8), cache) * st.V_scale[b, h].double()[at, None]
                q = st.q[b, h * G:(h + 1) * G].double()
                s = q @ k.T / math.sqrt(case["d"])
                if st.bias is not None:
                    s = s + st.bias[b, h, :n].double()
                if st.k is not None:
                    s = torch.cat([s, (q @ st.k[b, h].double() / math.sqrt(case["d"]))[:, None]], 1)
                    v = torch.cat([v, st.v[b, h].double()[None]])
                got["out"][b, h * G:(h + 1) * G] = torch.softmax(s, 1) @ v
        if st.k is None:
            return got
        k, v, counts, bias = st.k[:, :, None], st.v[:, :, None], [1] * case["batch"], None
    else:
        k, v, counts, bias = st.k, st.v, st.counts.tolist(), st.b
    tensors = dict(K=(st.K, st.K_scale, k), V=(st.V, st.V_scale, v))
    if sum(counts) / block > 20000:  # too many blocks for one at a time
        return None
    for name, (codes, scale, x) in tensors.items():
        values, scales = [], []
        for b, n in enumerate(lens):
            value, s = _exact_value(codes[b].view(torch.int8), cache), scale[b].double()
            _exact_store(value, s, x[b, :, :counts[b]], n, block, cache)
            values.append(value)
            scales.append(s)
        got[name], got[name + "_scale"] = torch.stack(values), torch.stack(scales)
    got["lengths"] = st.base + torch.tensor(counts, dtype=torch.int32, device="cuda")
    if st.bias is not None:
        full = st.bias.double()
        for b, n in enumerate(lens):
            full[b, :, n:n + counts[b]] = 0.0 if bias is None else bias[b, :, :counts[b]].double()
        got["bias"] = full
    return got
