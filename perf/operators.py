"""Operators around one decode step over the index, as cases to be timed.

  heads    dynakv_norm_rope: a layer's projected queries and keys are normed per head, rotated by their positions and
           laid out as the index takes them, the values with them
  pack     dynakv_packed_write and dynakv_packed_read: new entries are quantised into a packed cache and the same entries
           read back
  unpack   dynakv_packed_read: entries of a standing packed cache by position
  packed   dynakv_packed_attend: a tree of drafted tokens (one token: plain decoding) attends to a packed cache
  tree     dynakv_attend_tree: the same over the entries that the index's last retrieval gathered

The packed form of 32 neighbouring values of a row: codes of 8 or 4 bits (integers up to +-127 or +-7) and one scale 2^e,
held as the byte e + 127: the smallest e for which no code is cut off, within the range in which every code times 2^e is a
finite, exactly held value of the cache's type.  Codes of 4 bits lie two to a byte, the even one low.
"""
import math

import torch

own = False

D = 128                                   # head_dim, the one the library takes
BLOCK = 32                                # values that share a scale
COMP_STD, QUERY_NOISE, OUTLIERS, OUTLIER_SCALE = 0.3, 0.5, 4, 8.0      # the mixture of workload.py
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
QMAX = {8: 127, 4: 7}
E_RANGE = {("f16", 8): (-24, 9), ("f16", 4): (-24, 13), ("bf16", 8): (-126, 121), ("bf16", 4): (-126, 125),
           ("f32", 8): (-126, 121), ("f32", 4): (-126, 125)}


def _heads(name, dtype, seqs, tokens, kv_heads, group, rot=128, interleaved=False, norm=True, start=0, padded=False):
    return dict(name=name, kind="heads", dtype=dtype, seqs=seqs, tokens=tokens, kv_heads=kv_heads, group=group, rot=rot,
                interleaved=interleaved, norm=norm, start=start, padded=padded)


def _pack(name, dtype, bits, units, tokens, capacity):
    return dict(name=name, kind="pack", dtype=dtype, bits=bits, units=units, tokens=tokens, capacity=capacity)


def _unpack(name, dtype, bits, units, tokens, capacity):
    return dict(name=name, kind="unpack", dtype=dtype, bits=bits, units=units, tokens=tokens, capacity=capacity)


def _packed(name, dtype, bits, units, group, nodes, shortest, longest):
    return dict(name=name, kind="packed", dtype=dtype, bits=bits, units=units, group=group, nodes=nodes, shortest=shortest,
                longest=longest)


def _tree(name, dtype, units, group, nodes, tokens, clusters, budget):
    return dict(name=name, kind="tree", dtype=dtype, units=units, group=group, nodes=nodes, tokens=tokens, clusters=clusters,
                budget=budget)


def listed():
    return [
        # the smallest call: one sequence's next token, 8 KV heads of 4 query heads each, far into its context
        _heads("heads_one_token", "f16", 1, 1, 8, 4, start=12288),
        # a batch of 16 sequences with trees of up to 13 drafted tokens, ragged (padded rows are left as they are), half of
        # every head rotated, in neighbouring pairs
        _heads("heads_drafts_f32", "f32", 16, 13, 4, 7, rot=64, interleaved=True, start=30000, padded=True),
        # the longest prompt the index clusters at once, 8 KV heads of 8 query heads
        _heads("heads_prompt_bf16", "bf16", 1, 16384, 8, 8),
        # one decode step of 16 sequences x 8 KV heads: every unit writes its new entry and reads it back
        _pack("pack_step", "bf16", 8, 128, 1, 8192),
        # a prompt of 4096 tokens on 256 units (32 layers x 8 KV heads)
        _pack("pack_prompt", "f16", 4, 256, 4096, 4096),
        # a parked session comes back: everything is read, in the order of a snapshot's clusters
        _unpack("unpack_session", "bf16", 8, 112, 8192, 8192),
        # a retrieval's entries out of the longest context
        _unpack("unpack_selection", "f16", 4, 8, 4096, 131072),
        # plain decoding over a dense layer of the longest context: 8 units of 8 query heads, one token
        _packed("packed_decode_long", "bf16", 8, 8, 8, 1, 131072, 131072),
        # trees of 32 drafted tokens of 16 sequences x 8 KV heads whose caches differ in length
        _packed("packed_trees", "f16", 4, 128, 4, 32, 1, 8191),
        # the smallest configuration: float32, one unit, a chain of five drafted tokens over a budget of 256
        _tree("tree_tiny_f32", "f32", 1, 4, 5, 2048, 32, 256),
        # 32 layers x 8 KV heads, eight drafted tokens, budget 1024
        _tree("tree_llama3", "f16", 256, 4, 8, 4096, 256, 1024),
        # 28 layers x 4 KV heads of seven query heads, a wide tree of 61 nodes, budget 2048
        _tree("tree_qwen25_wide", "bf16", 112, 7, 61, 4096, 256, 2048),
    ]


def _log(rng, lo, hi):
    hi = max(lo, hi)
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["heads", "pack", "unpack", "packed", "packed", "tree", "tree"])
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    bits = rng.choice([8, 4])
    group = rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 12, 16])
    if kind == "heads":
        kv_heads = rng.choice([1, 2, 3, 4, 8])
        rows = (700000 if dtype == "f32" else 1300000) // (kv_heads * (group + 2))
        tokens = rng.choice([1, _log(rng, 1, 64), _log(rng, 64, 16384)])
        tokens = min(tokens, rows)
        seqs = _log(rng, 1, max(1, min(256, rows // tokens)))
        case = _heads("", dtype, seqs, tokens, kv_heads, group, rot=rng.choice([128, 128, 64, 96, 32, 8, 0]),
                      interleaved=rng.random() < 0.4, norm=rng.random() < 0.7, start=_log(rng, 1, 131072), padded=rng.random() < 0.5)
    elif kind in ("pack", "unpack"):
        units = _log(rng, 1, 256)
        tokens = _log(rng, 1, max(1, min(8192, (400000 if dtype == "f32" else 900000) // units)))
        case = (_pack if kind == "pack" else _unpack)("", dtype, bits, units, tokens, tokens + _log(rng, 1, 2048))
    elif kind == "packed":
        units, nodes = _log(rng, 1, 128), rng.choice([1, 1, rng.randint(1, 64)])
        if dtype == "f32":
            nodes = min(nodes, 16)
        most = min(131072, 1048576 // units, (1 << 24 if dtype == "f32" else 1 << 26) // (units * nodes * group))
        longest = _log(rng, 16, most)
        case = _packed("", dtype, bits, units, group, nodes, rng.choice([0, 1, longest // 2, longest]), longest)
    else:
        units, nodes = _log(rng, 1, 256), rng.randint(1, 64)
        if dtype == "f32":
            units, nodes = min(units, 32), min(nodes, 16)
        tokens = _log(rng, 700, 16384 if units <= 64 else 4096)
        clusters = max(16, int(tokens / rng.uniform(8, 24)))
        if dtype == "f32":
            clusters = min(clusters, 512)
        most = min(4096, tokens, (1 << 23 if dtype == "f32" else 1 << 26) // (units * nodes * group))
        case = _tree("", dtype, units, group, nodes, tokens, clusters, _log(rng, 256, most))
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------- inputs
def _trees(gen, units, nodes):
    """Ancestor bits [units, nodes] int64: node 0 is the root, every later one hangs on an earlier one, mostly a recent one;
    an eighth of the units has a shorter tree, whose padding nodes see no drafted token."""
    bits = torch.zeros(units, nodes, dtype=torch.int64, device="cuda")
    back = torch.rand(units, nodes, generator=gen, device="cuda").square()
    ids = torch.arange(units, device="cuda")
    for i in range(nodes):
        above = bits[ids, i - 1 - (back[:, i] * i).long().clamp_max(i - 1)] if i else 0
        bits[:, i] = above | (-(1 << 63) if i == 63 else 1 << i)
    count = torch.where(torch.rand(units, generator=gen, device="cuda") < 0.125,
                        torch.randint(1, nodes + 1, (units,), generator=gen, device="cuda"), nodes)
    return bits * (torch.arange(nodes, device="cuda")[None, :] < count[:, None])


def _channels(rnd, gen, units):
    chan = torch.ones(units, D, device="cuda")
    return chan.scatter_(1, torch.rand(units, D, generator=gen, device="cuda").topk(OUTLIERS, 1).indices, OUTLIER_SCALE)


def _cast(x, dt):
    return x.to(dt).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    ids = lambda n, *s: torch.randint(0, n, s, generator=gen, device="cuda")  # noqa: E731
    dt, kind = TYPES[case["dtype"]], case["kind"]
    s = dict(case=case)
    if own:
        from paper_2511_07427_amd import binding
        s["dynakv"] = binding
    if kind == "heads":
        B, T, H, G = case["seqs"], case["tokens"], case["kv_heads"], case["group"]
        # one projection's output holds the queries, keys and values of a token side by side
        fused = torch.empty(B, T, (H * G + 2 * H) * D, dtype=dt, device="cuda")
        for b in range(B):
            fused[b] = rnd(T, fused.shape[2]).to(dt)
        q, k, v = fused.split([H * G * D, H * D, H * D], dim=2)
        s["q"], s["k"], s["v"] = q.unflatten(2, (H * G, D)), k.unflatten(2, (H, D)), v.unflatten(2, (H, D))
        s["wq"], s["wk"] = ((1.0 + 0.2 * rnd(2, D)).to(dt) if case["norm"] else (None, None))
        s["freq"] = None
        if case["rot"]:
            s["freq"] = (500000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda").double() / case["rot"])).float()
        pos = case["start"] + ids(257, B, 1) + torch.arange(T, device="cuda")[None, :]
        if case["padded"]:
            pos = torch.where(torch.arange(T, device="cuda")[None, :] < 1 + ids(T, B, 1), pos, -1)
        s["pos"] = pos.int().contiguous()
        s["out"] = (torch.zeros(B * H, T, G, D, dtype=dt, device="cuda"), torch.zeros(B * H, T, D, dtype=dt, device="cuda"),
                    torch.zeros(B * H, T, D, dtype=dt, device="cuda"))
        return s
    U = case["units"]
    if kind in ("pack", "unpack", "packed"):
        n = case["tokens"] if kind == "pack" else case["longest"] if kind == "packed" else case["capacity"]
        cap = max(1, n if kind == "packed" else case["capacity"])
        chan = _channels(rnd, gen, U)
        K, V = torch.empty(U, n, D, dtype=dt, device="cuda"), torch.empty(U, n, D, dtype=dt, device="cuda")
        for u in range(0, U, 16):
            K[u:u + 16] = (rnd(min(16, U - u), n, D) * chan[u:u + 16, None, :]).to(dt)
            V[u:u + 16] = rnd(min(16, U - u), n, D).to(dt)
        width = D * case["bits"] // 8
        cache = [torch.zeros(U, cap, w, dtype=torch.uint8, device="cuda") for w in (width, D // BLOCK, width, D // BLOCK)]
        if kind == "pack":
            s["start"] = ids(cap - n + 1, U).int()
            s["positions"] = (s["start"][:, None] + torch.arange(n, device="cuda")[None, :]).int().contiguous()
            s["K"], s["V"] = K, V
        else:
            for u in range(0, U, 16):
                for x, at in ((K, 0), (V, 2)):
                    codes, scales = _quantise(x[u:u + 16], case)
                    cache[at][u:u + 16], cache[at + 1][u:u + 16] = codes, scales
            if kind == "unpack":
                s["positions"] = torch.rand(U, cap, generator=gen, device="cuda").argsort(1)[:, :case["tokens"]].int().contiguous()
        s["cache"] = cache
        if kind != "packed":
            s["out"] = tuple(torch.empty(U, case["tokens"], D, dtype=dt, device="cuda") for _ in range(2))
        else:
            span = torch.linspace(case["shortest"], n, U, device="cuda") if U > 1 else torch.full((1,), float(n), device="cuda")
            s["lengths"] = span.round().int()[torch.rand(U, generator=gen, device="cuda").argsort()].contiguous()
            # queries lie near one of the keys
            base = K[torch.arange(U, device="cuda"), ids(n, U)].float()
            queries, chan_new = base, chan
        if own:
            s["handle"] = s["dynakv"].PackedCache(*cache, dtype=case["dtype"])
    if kind == "tree":
        n, M = case["tokens"], case["clusters"]
        chan = _channels(rnd, gen, U)
        mean = rnd(U, M, D) * chan[:, None, :]
        label = ids(M, U, n)
        label[:, :M] = torch.arange(M, device="cuda")          # no cluster is empty
        K, V = torch.empty(U, n, D, dtype=dt, device="cuda"), torch.empty(U, n, D, dtype=dt, device="cuda")
        for u in range(0, U, 16):
            m = torch.gather(mean[u:u + 16], 1, label[u:u + 16, :, None].expand(-1, -1, D))
            K[u:u + 16] = (m + COMP_STD * rnd(*m.shape) * chan[u:u + 16, None, :]).to(dt)
            V[u:u + 16] = rnd(*m.shape).to(dt)
        size = torch.zeros(U, M, dtype=torch.int64, device="cuda").scatter_add_(1, label, torch.ones_like(label))
        queries, chan_new = K[torch.arange(U, device="cuda"), ids(n, U)].float(), chan
    if kind in ("packed", "tree"):
        T, G = case["nodes"], case["group"]
        s["Q"] = _cast(queries[:, None, None, :] + QUERY_NOISE * rnd(U, T, G, D), dt)
        s["K1"] = _cast(rnd(U, T, D) * chan_new[:, None, :], dt)
        s["V1"] = _cast(rnd(U, T, D), dt)
        s["tree"] = _trees(gen, U, T)
        s["out"] = torch.empty(U, T, G, D, dtype=dt, device="cuda")
        s["lse"] = torch.empty(U, T, G, dtype=torch.float32, device="cuda")
        if own:
            s["scratch"] = s["dynakv"].tree_scratch(U, T, G, "cuda:0")
    if kind == "packed":
        return s
    if kind == "tree":
        # the clusters that the root's queries select: by score, ties to the lower id, while their sizes fit the budget
        Q0 = s["Q"][:, 0].contiguous()
        score = torch.bmm(Q0.double(), mean.to(dt).double().transpose(1, 2).contiguous()).amax(1)
        order = torch.sort(score, dim=1, descending=True, stable=True).indices
        fits = (torch.gather(size, 1, order).cumsum(1) <= case["budget"]).cummin(1).values
        taken = torch.zeros(U, M, dtype=torch.bool, device="cuda").scatter_(1, order, fits)
        there = torch.gather(taken, 1, label)
        s["valid"], at = there.int().sort(dim=1, descending=True, stable=True)
        s["valid"], s["at"] = s["valid"][:, :case["budget"]].bool().contiguous(), at[:, :case["budget"]].contiguous()
        s["K"], s["V"] = K, V
        if own:
            binding = s["dynakv"]
            s["handle"] = binding.Index(binding.Config(U, case["group"], case["dtype"], M, M, n))
            zero = torch.zeros(U, M, dtype=torch.int32, device="cuda")
            offsets = torch.zeros(U, M + 1, dtype=torch.int32, device="cuda")
            offsets[:, 1:] = size.cumsum(1)
            s["handle"].dynakv_import_state(dict(
                n_clusters=torch.full((U,), M, dtype=torch.int32, device="cuda"),
                n_tokens=torch.full((U,), n, dtype=torch.int32, device="cuda"),
                tau=torch.full((U,), 1e9, dtype=torch.float64, device="cuda"), centroids=mean.contiguous(), size=size.int(),
                buffered=zero, flag=zero, m2=size.double(), offsets=offsets,
                members=label.argsort(dim=1, stable=True).int().contiguous(), keys=K, values=V))
            s["handle"].dynakv_retrieve_attend(Q0, case["budget"], torch.empty(U, case["group"], D, device="cuda"), None)
            torch.cuda.synchronize()
        return s
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _two_to(e):
    """2^e as float32 for integers e in -126..127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x, case):
    """Codes (two to a byte where they have four bits) and scale bytes of x [..., D]."""
    qmax, (lo, hi) = QMAX[case["bits"]], E_RANGE[case["dtype"], case["bits"]]
    b = x.float().unflatten(-1, (D // BLOCK, BLOCK))
    amax = b.abs().amax(-1)
    k = (amax.view(torch.int32) >> 23) - 127                       # amax lies in [2^k, 2^(k+1))
    e = (k - (6 if qmax == 127 else 2)).clamp(lo, hi)
    e = (e + (amax > qmax * _two_to(e))).clamp_max(hi)
    c = (b * _two_to(-e)[..., None]).round().clamp(-qmax, qmax).to(torch.int32).flatten(-2)
    scales = (e + 127).to(torch.uint8)
    if case["bits"] == 4:
        c = (c[..., 0::2] & 15) | ((c[..., 1::2] & 15) << 4)
    return (c & 255).to(torch.uint8), scales


def _values(codes, scales, case):
    c = codes.to(torch.int32)
    if case["bits"] == 4:
        c = torch.stack((c & 15, c >> 4), dim=-1).flatten(-2)
        c = torch.where(c > 7, c - 16, c)
    else:
        c = torch.where(c > 127, c - 256, c)
    e = scales.to(torch.int32) - 127
    return (c.float().unflatten(-1, (D // BLOCK, BLOCK)) * _two_to(e)[..., None]).flatten(-2)


def _rotate(x, cos, sin, case):
    h = case["rot"] // 2
    if h == 0:
        return x
    r, rest = x[..., :2 * h], x[..., 2 * h:]
    if case["interleaved"]:
        a, b = r[..., 0::2], r[..., 1::2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = r[..., :h], r[..., h:]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((y, rest), dim=-1)


def _normed(x, w):
    x = x.float()
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()


def _plain_heads(s):
    case = s["case"]
    B, T, H, G = case["seqs"], case["tokens"], case["kv_heads"], case["group"]
    dt, pos = TYPES[case["dtype"]], s["pos"]
    cos = sin = None
    if case["rot"]:
        angle = pos.double()[:, :, None] * s["freq"].double()
        cos, sin = angle.cos().float()[:, :, None, :], angle.sin().float()[:, :, None, :]
    there = (pos >= 0)[:, None, :, None]
    q = _rotate(_normed(s["q"], s["wq"]), cos, sin, case).unflatten(2, (H, G)).permute(0, 2, 1, 3, 4)
    k = _rotate(_normed(s["k"], s["wk"]), cos, sin, case).permute(0, 2, 1, 3)
    v = s["v"].permute(0, 2, 1, 3)
    # rows without a position keep what the outputs held: zeros
    return (torch.where(there[..., None], q, 0.0).to(dt).reshape(B * H, T, G, D),
            torch.where(there, k, 0.0).to(dt).reshape(B * H, T, D),
            torch.where(there, v, torch.zeros((), dtype=dt, device=v.device)).reshape(B * H, T, D))


def _plain_attend(s, K, V, valid):
    """softmax over the cache's entries (K, V [U, L, D] float32, valid [U, L]) and each node's ancestors."""
    case = s["case"]
    U, T, G = case["units"], case["nodes"], case["group"]
    Q = s["Q"].float().reshape(U, T * G, D)
    seen = ((s["tree"][:, :, None] >> torch.arange(T, device="cuda")) & 1).bool()                    # [U, node, drafted token]
    scale = 1.0 / math.sqrt(D)
    a = torch.bmm(Q, K.transpose(1, 2).contiguous()).mul_(scale).masked_fill_(~valid[:, None, :], -math.inf)
    b = torch.bmm(Q, s["K1"].float().transpose(1, 2).contiguous()).mul_(scale)
    b = b.masked_fill_(~seen.repeat_interleave(G, dim=1), -math.inf)
    m = b.amax(-1)
    if a.shape[2]:
        m = torch.maximum(m, a.amax(-1))
    none = m == -math.inf                                                                            # a row that sees nothing
    m = torch.where(none, 0.0, m)[..., None]
    a, b = a.sub_(m).exp_(), b.sub_(m).exp_()
    den = (a.sum(-1) + b.sum(-1))
    out = (torch.bmm(a, V) + torch.bmm(b, s["V1"].float())) / torch.where(none, 1.0, den)[..., None]
    lse = torch.where(none, -math.inf, m[..., 0] + den.log())
    return {"out": out.to(TYPES[case["dtype"]]).reshape(U, T, G, D), "lse": lse.reshape(U, T, G)}


def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "heads":
        return _plain_heads(s)
    dt = TYPES[case["dtype"]]
    if kind == "pack":
        rows = torch.arange(case["units"], device="cuda")[:, None], s["positions"].long()
        kc, ks, vc, vs = s["cache"]
        for x, codes, scales in ((s["K"], kc, ks), (s["V"], vc, vs)):
            codes[rows], scales[rows] = _quantise(x, case)
        return _values(kc[rows], ks[rows], case).to(dt), _values(vc[rows], vs[rows], case).to(dt)
    if kind == "unpack":
        rows = torch.arange(case["units"], device="cuda")[:, None], s["positions"].long()
        kc, ks, vc, vs = (x[rows] for x in s["cache"])
        return _values(kc, ks, case).to(dt), _values(vc, vs, case).to(dt)
    if kind == "packed":
        kc, ks, vc, vs = s["cache"]
        valid = torch.arange(kc.shape[1], device="cuda")[None, :] < s["lengths"][:, None]
        return _plain_attend(s, _values(kc, ks, case), _values(vc, vs, case), valid)
    at = s["at"][:, :, None].expand(-1, -1, D)
    return _plain_attend(s, torch.gather(s["K"], 1, at).float(), torch.gather(s["V"], 1, at).float(), s["valid"])


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    if not own:
        return _plain(s)
    case, kind, out = s["case"], s["case"]["kind"], s["out"]
    if kind == "heads":
        s["dynakv"].dynakv_norm_rope(s["q"], s["k"], s["v"], s["pos"], *out, q_weight=s["wq"], k_weight=s["wk"], inv_freq=s["freq"],
                                     eps=1e-6, interleaved=case["interleaved"])
        return out
    if kind in ("pack", "unpack"):
        if kind == "pack":
            s["handle"].dynakv_packed_write(s["K"], s["V"], s["start"])
        s["handle"].dynakv_packed_read(s["positions"], *out)
        return out
    if kind == "packed":
        s["handle"].dynakv_packed_attend(s["lengths"], s["Q"], s["K1"], s["V1"], s["tree"], out, s["lse"], s["scratch"])
    else:
        s["handle"].dynakv_attend_tree(s["Q"], s["K1"], s["V1"], s["tree"], out, s["lse"], s["scratch"])
    return {"out": out, "lse": s["lse"]}


def work(case):
    """Each input read once, each output written once; attention: two products of every row with every entry."""
    e = 4 if case["dtype"] == "f32" else 2
    kind = case["kind"]
    if kind == "heads":
        rows = case["seqs"] * case["tokens"] * case["kv_heads"] * (case["group"] + 2)
        if case["padded"]:
            rows = rows * (case["tokens"] + 1) // (2 * case["tokens"])       # about half the rows of a ragged batch
        return {"bytes": rows * 2 * D * e + case["seqs"] * case["tokens"] * 4, "flops": 8.0 * rows * D}
    U = case["units"]
    row, packed = 2 * D * e, 2 * (D * case["bits"] // 8 + D // BLOCK) if "bits" in case else 0
    if kind == "pack":
        return {"bytes": U * case["tokens"] * (2 * row + 2 * packed + 4) + 4 * U, "flops": 6.0 * U * case["tokens"] * 2 * D}
    if kind == "unpack":
        return {"bytes": U * case["tokens"] * (row + packed + 4), "flops": 2.0 * U * case["tokens"] * 2 * D}
    R, T = case["nodes"] * case["group"], case["nodes"]
    if kind == "packed":
        entries = U * (case["shortest"] + case["longest"]) / 2.0 if U > 1 else case["longest"]
        per = packed
    else:
        # a selection ends about half a cluster below the budget
        entries = U * min(case["tokens"], max(1.0, case["budget"] - 0.5 * case["tokens"] / case["clusters"]))
        per = row + 4
    moved = entries * per + U * (T * (row + 8) + R * (2 * D * e + 4))
    return {"bytes": moved, "flops": 4.0 * D * R * (entries + U * T / 2.0)}


# ---------------------------------------------------------------------------------------------- the definition in 64 bits
def _step64(e):
    """2^e in float64."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_pack(x, case):
    qmax, (lo, hi) = QMAX[case["bits"]], E_RANGE[case["dtype"], case["bits"]]
    y = x.double().reshape(*x.shape[:-1], D // BLOCK, BLOCK)
    ladder = qmax * _step64(torch.arange(lo, hi + 1, device=x.device))      # the largest value that each scale can hold
    e = lo + torch.searchsorted(ladder, y.abs().amax(-1, keepdim=True)).clamp_max(hi - lo)
    return ((y * _step64(-e)).round().clamp(-qmax, qmax) * _step64(e)).reshape(x.shape)


def _exact_unpack(codes, scales, case):
    if case["bits"] == 8:
        c = codes.view(torch.int8).double()
    else:
        c = torch.empty(*codes.shape[:-1], D, dtype=torch.float64, device=codes.device)
        c[..., 0::2], c[..., 1::2] = (codes & 15).double(), (codes >> 4).double()
        c -= 16.0 * (c >= 8)
    return c * _step64(scales.long() - 127).repeat_interleave(BLOCK, -1)


def _exact_attend(s, u, K, V):
    case = s["case"]
    T, G = case["nodes"], case["group"]
    keys, values = torch.cat((K, s["K1"][u].double())), torch.cat((V, s["V1"][u].double()))
    bits = s["tree"][u]
    seen = torch.stack([(bits >> j) & 1 for j in range(T)], 1) == 1
    seen = torch.cat((torch.ones(T, K.shape[0], dtype=torch.bool, device="cuda"), seen), 1)[:, None, :]
    logits = torch.where(seen, s["Q"][u].double() @ keys.T / D ** 0.5, -math.inf)
    lse = torch.logsumexp(logits, -1)
    p = torch.where(seen, (logits - torch.where(lse == -math.inf, 0.0, lse)[..., None]).exp(), 0.0)
    return p @ values, lse


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "heads":
        G, H = case["group"], case["kv_heads"]
        q, k, v = torch.zeros_like(s["out"][0], dtype=torch.float64), *(torch.zeros_like(s["out"][1], dtype=torch.float64) for _ in range(2))

        def turned(x, w, pos):
            if w is not None:
                x = x / (x.pow(2).sum(-1, keepdim=True) / D + 1e-6).sqrt() * w.double()
            h = case["rot"] // 2
            if h:
                z = (torch.complex(x[..., 0:2 * h:2], x[..., 1:2 * h:2]) if case["interleaved"] else torch.complex(x[..., :h], x[..., h:2 * h]))
                angle = pos.double()[:, None, None] * s["freq"].double()
                z = z * torch.complex(angle.cos(), angle.sin())
                y = torch.stack((z.real, z.imag), -1).flatten(-2) if case["interleaved"] else torch.cat((z.real, z.imag), -1)
                x = torch.cat((y, x[..., 2 * h:]), -1)
            return x

        for b in range(case["seqs"]):
            rows = torch.nonzero(s["pos"][b] >= 0)[:, 0]
            pos, units = s["pos"][b, rows], slice(b * H, (b + 1) * H)
            q[units, rows] = turned(s["q"][b, rows].double(), s["wq"], pos).reshape(-1, H, G, D).transpose(0, 1)
            k[units, rows] = turned(s["k"][b, rows].double(), s["wk"], pos).transpose(0, 1)
            v[units, rows] = s["v"][b, rows].double().transpose(0, 1)
        return q, k, v
    if kind == "pack":
        return _exact_pack(s["K"], case), _exact_pack(s["V"], case)
    U = case["units"]
    if kind == "unpack":
        got = []
        for c, e in (s["cache"][:2], s["cache"][2:]):
            got.append(torch.stack([_exact_unpack(c[u, s["positions"][u].long()], e[u, s["positions"][u].long()], case) for u in range(U)]))
        return tuple(got)
    out, lse = [], []
    for u in range(U):
        if kind == "packed":
            n = int(s["lengths"][u])
            kc, ks, vc, vs = (x[u, :n] for x in s["cache"])
            o, l = _exact_attend(s, u, _exact_unpack(kc, ks, case), _exact_unpack(vc, vs, case))
        else:
            at = s["at"][u][s["valid"][u]]
            o, l = _exact_attend(s, u, s["K"][u, at].double(), s["V"][u, at].double())
        out.append(o)
        lse.append(l)
    return {"out": torch.stack(out), "lse": torch.stack(lse)}
