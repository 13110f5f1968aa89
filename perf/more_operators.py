"""The operators of a speculative step over a compressed cache as measurable cases: rotary positions of
queries and keys, attention of a tree of drafted tokens over the cache, verification of the drafts against
the target's probabilities, and the accepted path's rows put into the caches of a model's layers.

A pass is one call of `paper_2607_16213_gb300.api` on device tensors (`rotary`, `tree_attn`,
`tree_verify`, `tree_commit`), with the caches, the plan and the workspace kept across calls as a serving program
keeps them.  A pass that commits first puts the lengths back to where the case starts, as a program does that
tries another continuation; the rows written before are written over.

A tree: T tokens of a sequence, token 0 the last one that is certain (its row is not in the cache yet), every
other token's parent before it.  A token sees the cache, its ancestors and itself.

Verification walks from token 0.  At a node with target distribution p and draft distribution q the weights are
r = p with mass M = 1; its children are tried in order: token x is accepted where u M q(x) < r(x), else
r becomes max(r - M q, 0) and M the sum of that.  Drafts picked without drawing (no q): accepted where
u M < r(x), else r(x) becomes 0 and M loses it.  Where no child is accepted, the next token is drawn from r: the first one
whose running sum passes u0 times the whole.  Token t's own number decides on it, that of token 0 draws.
"""
import math

import torch

own = False

_LLAMA = dict(dtype="bf16", hq=32, hkv=8, d=128)
_SMALL = dict(dtype="fp32", hq=4, hkv=2, d=64)


def listed():
    def rotary(name, batch, tokens, far, layout, rot, scaling, shape=_LLAMA):
        return dict(name=name, kind="rotary", batch=batch, tokens=tokens, far=far, layout=layout, rot=rot, scaling=scaling,
                    theta=10000.0, **shape)

    def attn(name, batch, rows, tokens, shape=_LLAMA, ragged=False, bias=True, chain=False):
        return dict(name=name, kind="attn", batch=batch, rows=rows, tokens=tokens, ragged=ragged, bias=bias, chain=chain, **shape)

    def verify(name, batch, tokens, vocab, drawn, ragged=False):
        return dict(name=name, kind="verify", batch=batch, tokens=tokens, vocab=vocab, drawn=drawn, ragged=ragged)

    def commit(name, layers, batch, rows, tokens, shape=_LLAMA, bias=True):
        return dict(name=name, kind="commit", layers=layers, batch=batch, rows=rows, tokens=tokens, bias=bias, **shape)

    return [
        # a small tree of one sequence, positions behind a long prompt: latency
        rotary("rotary_t8", 1, 8, 100000, "half", 128, "wavelength"),
        # a long prompt before its scoring
        rotary("rotary_prompt_16k", 1, 16384, 16384, "interleaved", 128, "none"),
        # a small fp32 model's tree over an odd number of rows: latency
        attn("attn_fp32_t7", 2, 201, 7, _SMALL, ragged=True),
        # a short chain of drafts in the long-context setting (a 100k prompt at 25%)
        attn("attn_25k_t4", 1, 25000, 4, chain=True),
        # a tree of the same setting
        attn("attn_25k_t32", 1, 25000, 32),
        # small trees of a large ragged batch over short caches
        attn("attn_b64_819_t9", 64, 819, 9, ragged=True),
        # trees of eight ragged long caches
        attn("attn_b8_16k_t25", 8, 16384, 25, ragged=True),
        # a wide tree over an uncompressed cache without compensation, the largest case
        attn("attn_131k_t64_plain", 1, 131072, 64, bias=False),
        # one sequence's tree, drafts drawn from the draft's distribution: latency
        verify("verify_b1_32k", 1, 8, 32000, True),
        # the trees of a large ragged batch over a large vocabulary
        verify("verify_b64_128k", 64, 16, 128000, True, ragged=True),
        # one sequence's path into the caches of 32 layers
        commit("commit_l32_b1", 32, 1, 4096, 32),
        # a batch's paths into the caches of eight layers
        commit("commit_l8_b16", 8, 16, 819, 16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: batches of up to 64, trees of 1 to 64 tokens (verified: 32), caches of 40 to 131072 rows (at most 1M rows of
    all sequences and heads), vocabularies of 100 to 200000, up to 32 layers, both types."""
    kind = rng.choice(("rotary", "attn", "attn", "attn", "verify", "commit"))
    fp32 = rng.random() < 0.25
    hq, hkv = rng.choice(((32, 8), (32, 8), (64, 8), (32, 32), (32, 4), (32, 2)))
    if fp32 and rng.random() < 0.7:
        hq, hkv = 4, 2
    d = rng.choice((128, 128, 64))
    batch = rng.choice((1, 1, 2, 5, 8, 16, 33, 64))
    tokens = _log_int(rng, 1, 64)
    case = dict(kind=kind, batch=batch, tokens=tokens, dtype="fp32" if fp32 else "bf16", hq=hq, hkv=hkv, d=d)
    ragged = rng.random() < 0.7
    if kind == "rotary":
        most = 80000000 // ((hq + hkv) * d * batch * (2 if fp32 else 1))
        case.update(tokens=_log_int(rng, 1, max(2, most)), far=_log_int(rng, 100, 1000000), layout=rng.choice(("half", "interleaved")),
                    rot=d if rng.random() < 0.6 else rng.choice((16, 32, d // 2, d - 16)),
                    scaling=rng.choice(("none", "linear", "wavelength", "ramp")), theta=rng.choice((10000.0, 500000.0, 1e6)))
        return case
    if kind == "verify":
        tokens = min(tokens, 32)
        vocab = _log_int(rng, 100, min(200000, 120000000 // (batch * tokens)))
        return dict(kind=kind, batch=batch, tokens=tokens, vocab=vocab, drawn=rng.random() < 0.7, ragged=ragged)
    if kind == "commit":
        layers = rng.randint(1, max(1, min(32, 100000000 // (batch * hkv * d * (tokens + 64)))))
        most = max(41, 100000000 // (layers * batch * hkv * d))
        return dict(case, layers=layers, rows=_log_int(rng, 40, min(16384, most)), bias=rng.random() < 0.8)
    most = (100000 if fp32 else 1000000) // (batch * hkv)
    if hq // hkv > 4:  # (no more products than the largest listed case)
        most = most * 4 // (hq // hkv)
    return dict(case, rows=_log_int(rng, 40, max(41, min(131072, most))), ragged=ragged, bias=rng.random() < 0.8, chain=rng.random() < 0.3)


# ---- inputs ----------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _ragged(case, n):
    """Per sequence all n, or from about half of them up; of the case's sizes alone."""
    if not case.get("ragged") or n < 2:
        return [n] * case["batch"]
    lo = (n + 1) // 2
    return [lo + ((i * 2654435761 + 12345) % 1000003) * (n - lo + 1) // 1000003 for i in range(case["batch"])]


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _rows(g, B, H, n, d, dtype, keys):
    """Rows [B][H][n][d] in segments of 16 around random centroids; of keys 1% of the positions four times
    larger, 3% of the channels eight times."""
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


def _parents(seed, B, T, chain):
    """Token 0 the root; another one follows the token before it half the time, else any before it."""
    g = torch.Generator()
    g.manual_seed(int(seed) + 77)
    t = torch.arange(T)
    any_before = (torch.rand((B, T), generator=g) * t).long().clamp(max=max(0, T - 1))
    before = (torch.rand((B, T), generator=g) < 0.5) | chain
    p = torch.where(before, t - 1, any_before)
    p[:, 0] = -1
    return p.int().cuda()


class _State:
    def __init__(self, case, seed):
        self.case = case
        self.handle = None
        g = torch.Generator(device="cuda")
        g.manual_seed(int(seed))
        getattr(self, "_" + case["kind"])(case, g, seed)

    def _rotary(self, c, g, seed):
        B, T, d = c["batch"], c["tokens"], c["d"]
        base = torch.randint(0, max(1, c["far"] - T + 1), (B, 1), generator=g, device="cuda")
        self.positions = (base + torch.arange(T, device="cuda")).int()
        self.q = torch.randn((B, c["hq"], T, d), generator=g, device="cuda").to(_dtype(c))
        self.k = torch.randn((B, c["hkv"], T, d), generator=g, device="cuda").to(_dtype(c))
        self.q_out, self.k_out = torch.zeros_like(self.q), torch.zeros_like(self.k)

    def _attn(self, c, g, seed):
        B, H, T, d, n = c["batch"], c["hkv"], c["tokens"], c["d"], c["rows"]
        self.cap = (n + 63) // 64 * 64
        self.K, self.V = (_rows(g, B, H, self.cap, d, _dtype(c), keys) for keys in (True, False))
        self.bias = _bias(g, B, H, self.cap) if c["bias"] else None
        self.lengths, self.counts = _ints(_ragged(c, n)), _ints(_ragged(c, T))
        self.parents = _parents(seed, B, T, c["chain"])
        self.q = torch.randn((B, c["hq"], T, d), generator=g, device="cuda").to(_dtype(c))
        self.k, self.v = (torch.randn((B, H, T, d), generator=g, device="cuda").to(_dtype(c)) for _ in range(2))
        self.out = torch.zeros_like(self.q)

    def _verify(self, c, g, seed):
        B, T, V = c["batch"], c["tokens"], c["vocab"]
        self.parents, self.counts = _parents(seed, B, T, False), _ints(_ragged(c, T))
        self.uniforms = torch.rand((B, T), generator=g, device="cuda")
        self.tokens = torch.zeros((B, T), dtype=torch.int32, device="cuda")
        self.target = torch.empty((B, T, V), device="cuda")
        self.draft = torch.empty((B, T, V), device="cuda") if c["drawn"] else None
        pick = torch.rand((B, T), generator=g, device="cuda")
        for b in range(B):
            logits = torch.randn((T, V), generator=g, device="cuda").mul_(5.0)
            self.target[b] = torch.softmax(logits, 1)
            q = torch.softmax(logits.add_(torch.randn((T, V), generator=g, device="cuda"), alpha=0.7), 1)
            up = self.parents[b].long().clamp_min(0)
            if c["drawn"]:
                self.draft[b] = q
                cum = q.cumsum(1)[up]
                self.tokens[b] = torch.searchsorted(cum, (pick[b] * cum[:, -1])[:, None], right=True)[:, 0].clamp_max(V - 1).int()
            else:  # the children of a node: its most likely tokens in order
                rank = ((up[:, None] == up) & (torch.arange(T, device="cuda")[:, None] > torch.arange(T, device="cuda"))).sum(1)
                self.tokens[b] = q.topk(min(T, V), 1).indices[up, rank.clamp_max(V - 1)].int()

    def _commit(self, c, g, seed):
        L, B, H, T, d, n = c["layers"], c["batch"], c["hkv"], c["tokens"], c["d"], c["rows"]
        self.cap = (n + T + 63) // 64 * 64
        # the caches and the new rows of all layers side by side
        make = lambda rows: torch.stack([torch.randn((B, H, rows, d), generator=g, device="cuda").to(_dtype(c)) for _ in range(L)])  # noqa: E731
        self.K, self.V, self.k, self.v = make(self.cap), make(self.cap), make(T), make(T)
        self.bias = torch.stack([_bias(g, B, H, self.cap) for _ in range(L)]) if c["bias"] else None
        # (each layer's lengths 16-byte aligned)
        self.lengths = torch.full((L, (B + 3) // 4 * 4), n, dtype=torch.int32, device="cuda")
        self.base = self.lengths.clone()
        accepted = torch.randint(1, T + 1, (B,), generator=g, device="cuda")
        steps = torch.rand((B, T), generator=g, device="cuda").argsort(1)  # `accepted` of the tokens, in order
        live = torch.arange(T, device="cuda") < accepted[:, None]
        self.path = torch.where(live, torch.where(live, steps, T).sort(1).values, -1).int()
        self.accepted = accepted.int()


def prepare(case, seed):
    return _State(case, seed)


# ---- the plain forms -------------------------------------------------------------------------
_FACTOR, _ORIGINAL = 8.0, 8192
_BLEND = {"wavelength": (1.0, 4.0), "ramp": (1.0, 32.0)}


def _frequencies(c):
    """Radians a position of each pair (64 bits), and what cosine and sine are multiplied by."""
    rot, theta = c["rot"], c["theta"]
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    f = theta ** (-2.0 * i / rot)
    if c["scaling"] == "none":
        return f, 1.0
    if c["scaling"] == "linear":
        return f / _FACTOR, 1.0
    low, high = _BLEND[c["scaling"]]
    if c["scaling"] == "wavelength":  # by the turns that a pair makes over the original context
        keep = ((_ORIGINAL * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        return f * keep + f / _FACTOR * (1 - keep), 1.0
    at = lambda turns: rot * math.log(_ORIGINAL / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
    first, last = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot - 1)
    scaled = ((i - first) / max(last - first, 0.001)).clamp(0, 1)
    return f * (1 - scaled) + f / _FACTOR * scaled, 0.1 * math.log(_FACTOR) + 1.0


def _turn(x, cos, sin, c):
    rot = c["rot"]
    y = x.float().clone()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if c["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    u, v = x[..., a].float(), x[..., b].float()
    y[..., a], y[..., b] = u * cos - v * sin, v * cos + u * sin
    return y.to(x.dtype)


def _rotary(st):
    f, amplitude = _frequencies(st.case)
    angle = st.positions.double()[..., None] * f
    cos, sin = ((amplitude * fn(angle)).float()[:, None] for fn in (torch.cos, torch.sin))
    st.q_out.copy_(_turn(st.q, cos, sin, st.case))
    st.k_out.copy_(_turn(st.k, cos, sin, st.case))


def _sees(parents):
    """[B][T][T]: u is t or an ancestor of t; paths of doubling length by products."""
    T = parents.shape[1]
    step = (parents[..., None] == torch.arange(T, device="cuda")).float() + torch.eye(T, device="cuda")
    for _ in range(max(1, (T - 1).bit_length())):
        step = (step @ step).clamp_max(1.0)
    return step > 0


def _attn(st):
    B, Hq, T, d = st.q.shape
    H = st.K.shape[1]
    q = st.q.float().view(B, H, Hq // H * T, d) / math.sqrt(d)
    live = torch.arange(st.cap, device="cuda") < st.lengths[:, None]
    K, V = (torch.where(live[:, None, :, None], x.float(), 0.0) for x in (st.K, st.V))
    s = q @ K.transpose(2, 3)
    if st.bias is not None:
        s = s + st.bias[:, :, None]
    s = s.masked_fill(~live[:, None, None], -math.inf)
    sees = _sees(st.parents) & (torch.arange(T, device="cuda") < st.counts[:, None])[:, None]
    t = (q @ st.k.float().transpose(2, 3)).view(B, H, Hq // H, T, T).masked_fill(~sees[:, None, None], -math.inf)
    p = torch.cat([s, t.view(B, H, -1, T)], 3)
    m = p.amax(3, keepdim=True)
    p = torch.exp(p - torch.where(m == -math.inf, 0.0, m))
    z = p.sum(3, keepdim=True)
    o = (p @ torch.cat([V, st.v.float()], 2) / torch.where(z > 0, z, 1.0)).view(B, Hq, T, d)
    asked = (torch.arange(T, device="cuda") < st.counts[:, None])[:, None, :, None]
    st.out.copy_(torch.where(asked, o.to(st.out.dtype), st.out))


def _verify(st):
    """All sequences token by token (a token's parent is before it), weights in 64 bits: a number drawn may lie next to
    the border of two tokens."""
    B, T, V = st.target.shape
    at = torch.arange(B, device="cuda")
    tokens, parents, u = st.tokens.long(), st.parents.long(), st.uniforms.double()
    node = torch.zeros(B, dtype=torch.long, device="cuda")
    r, M = st.target[:, 0].double(), torch.ones(B, dtype=torch.float64, device="cuda")
    accepted = (st.counts > 0).int()
    path = torch.full((B, T + 1), -1, dtype=torch.int32, device="cuda")
    path[:, 0] = accepted - 1
    for t in range(1, T):
        x = tokens[:, t]
        tried = (parents[:, t] == node) & (t < st.counts)
        weight = r[at, x]
        if st.draft is not None:
            q = st.draft[at, node].double()
            yes = tried & (u[:, t] * M * q[at, x] < weight)
            left = (r - M[:, None] * q).clamp_min(0.0)
            mass = left.sum(1)
        else:
            yes = tried & (u[:, t] * M < weight)
            left = r.scatter(1, x[:, None], 0.0)
            mass = M - weight
        no = tried & ~yes & (mass > 0)
        r, M = torch.where(no[:, None], left, r), torch.where(no, mass, M)
        node, r = torch.where(yes, t, node), torch.where(yes[:, None], st.target[:, t].double(), r)
        M = torch.where(yes, 1.0, M)
        path.scatter_(1, torch.where(yes, accepted, T)[:, None].long(), t)
        accepted = accepted + yes.int()
    cum = r.cumsum(1)
    drawn = torch.searchsorted(cum, (u[:, :1] * cum[:, -1:]), right=True)[:, 0].clamp_max(V - 1).int()
    return dict(accepted=accepted, path=path[:, :T].contiguous(), next_token=torch.where(accepted > 0, drawn, -1))


def _commit(st):
    B, T = st.path.shape
    b, i = torch.nonzero(torch.arange(T, device="cuda") < st.accepted[:, None], as_tuple=True)
    src = st.path[b, i].long()
    to = st.lengths[:, b].long() + i
    layer = torch.arange(st.K.shape[0], device="cuda")[:, None].expand_as(to)
    b = b.expand_as(to)
    st.K[layer, b, :, to], st.V[layer, b, :, to] = st.k[layer, b, :, src.expand_as(to)], st.v[layer, b, :, src.expand_as(to)]
    if st.bias is not None:
        st.bias[layer, b, :, to] = 0.0
    st.lengths[:, :B] += st.accepted


# ---- one pass --------------------------------------------------------------------------------
def _handle(st):
    """What a program makes once: the plan, or the framework's caches over the state's tensors and a workspace."""
    import paper_2607_16213_gb300 as S
    from paper_2607_16213_gb300 import api
    c, kind = st.case, st.case["kind"]
    if kind == "rotary":
        shape = api.make_shape(c["dtype"], c["batch"], c["hq"], c["hkv"], c["d"], 32, 64, 64)
        scaling = {} if c["scaling"] == "none" else dict(scaling=c["scaling"], factor=_FACTOR)
        if c["scaling"] in _BLEND:
            low, high = _BLEND[c["scaling"]]
            scaling.update(original=_ORIGINAL, low=low, high=high)
        return api, shape, api.rotary_plan(c["rot"], c["theta"], c["layout"], **scaling)
    if kind == "verify":
        return api, None, api.Workspace(S.selkv_tree_verify_workspace_size(c["batch"], c["tokens"], c["vocab"]))
    shape = api.make_shape(c["dtype"], c["batch"], c["hq"], c["hkv"], c["d"], 32, st.cap, st.cap)
    if kind == "attn":
        bias = st.bias if st.bias is not None else torch.zeros((c["batch"], c["hkv"], st.cap), device="cuda")
        cache = api.CompressedCache(shape, st.K, st.V, bias, st.lengths)
        return api, cache, api.Workspace(S.selkv_tree_attn_workspace_size(shape, c["tokens"]))
    caches = [api.CompressedCache(shape, st.K[i], st.V[i], st.bias[i] if st.bias is not None else None, st.lengths[i, :c["batch"]])
              for i in range(c["layers"])]
    return api, caches, api.Workspace(S.selkv_tree_commit_workspace_size(shape))


def _own(st):
    if st.handle is None:
        st.handle = _handle(st)
    api, a, b = st.handle
    kind = st.case["kind"]
    if kind == "rotary":
        api.rotary(a, b, st.positions, st.q, st.k, out=(st.q_out, st.k_out))
    elif kind == "attn":
        api.tree_attn(a, st.q, st.k, st.v, st.parents, st.counts, use_bias=st.bias is not None, out=st.out, workspace=b)
    elif kind == "verify":
        accepted, path, next_token = api.tree_verify(st.tokens, st.parents, st.uniforms, st.target, st.draft, st.counts, workspace=b)
        return dict(accepted=accepted, path=path, next_token=next_token)
    else:
        api.tree_commit(a, list(st.k), list(st.v), st.path, st.accepted, workspace=b)


def run(st):
    kind = st.case["kind"]
    if kind == "commit":
        st.lengths.copy_(st.base)
    if own:
        got = _own(st)
    else:
        got = {"rotary": _rotary, "attn": _attn, "verify": _verify, "commit": _commit}[kind](st)
    if kind == "verify":
        return got
    if kind == "rotary":
        return dict(q=st.q_out, k=st.k_out)
    if kind == "attn":
        return dict(out=st.out)
    return dict(K=st.K, V=st.V, lengths=st.lengths, **({} if st.bias is None else dict(bias=st.bias)))


def work(case):
    e = 2 if case.get("dtype") == "bf16" else 4
    B, T = case["batch"], case["tokens"]
    if case["kind"] == "verify":
        # the distributions of a sequence's last node; a difference, a comparison and a sum of each weight
        rows = 2 if case["drawn"] else 1
        return dict(bytes=4 * B * case["vocab"] * rows + 16 * B * T, flops=(rows + 1.0) * B * case["vocab"])
    Hq, H, d = case["hq"], case["hkv"], case["d"]
    if case["kind"] == "rotary":
        return dict(bytes=2 * B * (Hq + H) * T * d * e + 4 * B * T, flops=3.0 * B * (Hq + H) * T * case["rot"])
    if case["kind"] == "commit":
        # half of a tree's tokens are accepted on the average
        rows = case["layers"] * B * H * (T + 1) / 2
        return dict(bytes=int(2 * 2 * rows * d * e + 4 * rows), flops=rows)
    rows, drafts = _ragged(case, case["rows"]), _ragged(case, T)
    by = (2 * H * d * e + (4 if case["bias"] else 0)) * sum(rows) + (2 * Hq + 2 * H) * d * e * sum(drafts) + 4 * B * T
    return dict(bytes=by, flops=4.0 * Hq * d * sum(t * (n + t) for n, t in zip(rows, drafts)))


# ---- the same in 64 bits ---------------------------------------------------------------------
def _exact_rotary(st):
    c = st.case
    rot, theta, n = c["rot"], c["theta"], st.positions.double()
    outs = []
    freqs, gain = [], 1.0
    for i in range(rot // 2):
        w = math.exp(-math.log(theta) * 2 * i / rot)
        s = 1.0  # share of the frequency that stays as it was
        if c["scaling"] == "linear":
            s = 0.0
        elif c["scaling"] == "wavelength":
            wave = 2 * math.pi / w
            low, high = _BLEND["wavelength"]
            s = 1.0 if wave < _ORIGINAL / high else 0.0 if wave > _ORIGINAL / low else (_ORIGINAL / wave - low) / (high - low)
        elif c["scaling"] == "ramp":
            slow, fast = _BLEND["ramp"]
            border = [rot / 2 * math.log(_ORIGINAL / (2 * math.pi * turns)) / math.log(theta) for turns in (fast, slow)]
            lo, hi = max(0, math.floor(border[0])), min(rot - 1, math.ceil(border[1]))
            s = 1.0 - min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            gain = 1.0 + 0.1 * math.log(_FACTOR)
        freqs.append(s * w + (1.0 - s) * w / _FACTOR)
    z = torch.polar(torch.full((rot // 2,), gain, dtype=torch.float64, device="cuda").expand(*n.shape, -1),
                    n[..., None] * torch.tensor(freqs, dtype=torch.float64, device="cuda"))[:, None]
    for x in (st.q, st.k):
        y = x.double()
        pair = y[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2) if c["layout"] == "half" else y[..., :rot].unflatten(-1, (rot // 2, 2))
        w = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * z)
        y[..., :rot] = (w.transpose(-1, -2) if c["layout"] == "half" else w).flatten(-2)
        outs.append(y)
    return dict(q=outs[0], k=outs[1])


def _exact_attn(st):
    c = st.case
    B, Hq, T, d = st.q.shape
    G = Hq // c["hkv"]
    out = torch.zeros(st.q.shape, dtype=torch.float64, device="cuda")
    parents = st.parents.tolist()
    for b, (n, m) in enumerate(zip(st.lengths.tolist(), st.counts.tolist())):
        sees = torch.zeros((m, m), dtype=torch.bool)
        for t in range(m):
            u = t
            while u >= 0:
                sees[t, u] = True
                u = parents[b][u]
        hidden = (~sees).cuda().repeat(G, 1)
        for h in range(c["hkv"]):
            q = st.q[b, h * G:(h + 1) * G, :m].double().reshape(G * m, d)
            s = q @ st.K[b, h, :n].double().T / math.sqrt(d)
            if st.bias is not None:
                s += st.bias[b, h, :n].double()
            s = torch.cat([s, (q @ st.k[b, h, :m].double().T / math.sqrt(d)).masked_fill(hidden, -math.inf)], 1)
            o = torch.softmax(s, 1) @ torch.cat([st.V[b, h, :n], st.v[b, h, :m]]).double()
            out[b, h * G:(h + 1) * G, :m] = o.view(G, m, d)
    return dict(out=out)


def _exact_verify(st):
    B, T, V = st.target.shape
    tokens, parents, u = st.tokens.tolist(), st.parents.tolist(), st.uniforms.double().tolist()
    accepted, path, drawn = [], [], []
    for b, m in enumerate(st.counts.tolist()):
        node, way = 0, [0]
        while True:
            p, mass, child = st.target[b, node].double(), 1.0, None
            q = st.draft[b, node].double() if st.draft is not None else None
            for t in [t for t in range(node + 1, m) if parents[b][t] == node]:
                x = tokens[b][t]
                if u[b][t] * mass * (float(q[x]) if q is not None else 1.0) < float(p[x]):
                    child = t
                    break
                if q is None:
                    if mass - float(p[x]) > 0:
                        mass -= float(p[x])
                        p[x] = 0.0
                else:
                    rest = torch.relu(p - mass * q)
                    if float(rest.sum()) > 0:
                        p, mass = rest, float(rest.sum())
            if child is None:
                break
            node = child
            way.append(child)
        run_sum = torch.cumsum(p, 0)
        drawn.append(min(V - 1, int((run_sum <= u[b][0] * float(run_sum[-1])).sum())))
        accepted.append(len(way))
        path.append(way + [-1] * (T - len(way)))
    return dict(accepted=_ints(accepted), path=_ints(path), next_token=_ints(drawn))


def _exact_commit(st):
    out = dict(K=st.K.double(), V=st.V.double(), lengths=st.base.clone())
    if st.bias is not None:
        out["bias"] = st.bias.double()
    path, start = st.path.tolist(), int(st.base[0, 0])
    out["lengths"][:, :len(path)] += st.accepted
    for b, a in enumerate(st.accepted.tolist()):
        out["K"][:, b, :, start:start + a] = st.k[:, b][:, :, path[b][:a]].double()
        out["V"][:, b, :, start:start + a] = st.v[:, b][:, :, path[b][:a]].double()
        if st.bias is not None:
            out["bias"][:, b, :, start:start + a] = 0.0
    return out


def exact(case, seed):
    st = _State(case, seed)
    return {"rotary": _exact_rotary, "attn": _exact_attn, "verify": _exact_verify, "commit": _exact_commit}[case["kind"]](st)
