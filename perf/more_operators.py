"""Performance cases of the operators around a pass behind the paged cache: norms
of queries and keys with the rotation in the same pass (and their gradient, and
the form that puts keys into their pages), attention of sequences that share a
prefix of pages, and the verification of drafted tokens.

The sizes are those of the repository's models and workloads (heads, vocabularies,
prompts, blocks), and longer contexts.  With `own` set, `run` calls the library;
without, it computes the same from elementary torch operations in float32 (angles,
long sums and what stands next to a border in float64).  `exact` computes a case
from its definition in float64, apart from both.
"""

from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # Queries and keys of a batch of prompts as one product gives them (a row:
        # queries, keys, values), for a context eight times as long as the trained one.
        dict(name="norm_prompts", kind="norm", rows=32768, heads=16, kv=4, hd=128, rot=128, layout="half",
             scaling="yarn", factor=8.0, original=4096, theta=10000.0, dtype="bf16", gain="bf16", far=32768),
        # One training step of the same: forward, and the gradients of queries, keys
        # and both gains, which are kept in float32.
        dict(name="norm_train", kind="train", rows=16384, heads=16, kv=4, hd=128, rot=128, layout="half",
             scaling="none", factor=1.0, original=0, theta=10000.0, dtype="bf16", gain="f32", far=4096),
        # An odd number of rows, interleaved pairs in a part of the head, float32.
        dict(name="norm_train_odd", kind="train", rows=4099, heads=16, kv=16, hd=64, rot=48, layout="interleaved",
             scaling="linear", factor=4.0, original=0, theta=10000.0, dtype="f32", gain="f32", far=16384),
        # One new token per sequence normalised, rotated and put into its page: a
        # decoding step of a batch, where latency is all.
        dict(name="put_tokens", kind="put", seqs=32, rows=1, heads=16, kv=4, hd=128, page=64, len_lo=64, len_hi=1024,
             dtype="bf16", src="bf16", gain="bf16", mix=1),
        # Ragged prompts put into their pages, straight from float32 products.
        dict(name="put_prompts", kind="put", seqs=32, rows=1024, heads=16, kv=4, hd=128, page=64, len_lo=0, len_hi=0,
             dtype="bf16", src="f32", gain="f32", mix=2),
        # One token of each of four continuations of a short prompt.
        dict(name="shared_few", kind="shared", layers=1, groups=1, members=4, alone=0, rows=1, ragged=False,
             mask="full", heads=16, kv=16, hd=64, page=16, prefix_lo=640, prefix_hi=640, tail_lo=1, tail_hi=64,
             dtype="bf16", mix=3),
        # A decoding step in four layers of a batch that answers one long document
        # in 64 ways.
        dict(name="shared_tokens", kind="shared", layers=4, groups=1, members=64, alone=0, rows=1, ragged=False,
             mask="full", heads=16, kv=4, hd=128, page=64, prefix_lo=16384, prefix_hi=16384, tail_lo=16, tail_hi=1024,
             dtype="bf16", mix=4),
        # The same of eight prompts with eight continuations each, and of sequences
        # that share nothing.
        dict(name="shared_groups", kind="shared", layers=4, groups=8, members=8, alone=6, rows=1, ragged=False,
             mask="full", heads=16, kv=4, hd=128, page=64, prefix_lo=1024, prefix_hi=8192, tail_lo=1, tail_hi=512,
             dtype="bf16", mix=5),
        # Trees of up to 13 drafted tokens of sixteen continuations of a long prompt.
        dict(name="shared_trees", kind="shared", layers=1, groups=1, members=16, alone=0, rows=13, ragged=True,
             mask="tree", heads=32, kv=8, hd=128, page=128, prefix_lo=32768, prefix_hi=32768, tail_lo=1, tail_hi=700,
             dtype="f16", mix=6),
        # Five drafted tokens of one sequence against the target, the draft's own
        # logits known.
        dict(name="verify_chain", kind="verify", seqs=1, rows=6, ragged=False, shape="chain", vocab=32768,
             dtype="f32", temperature=1.0, mix=7),
        # Chains of seven of a batch, the vocabulary of the large models.
        dict(name="verify_chains", kind="verify", seqs=32, rows=8, ragged=True, shape="chain", vocab=157184,
             dtype="bf16", temperature=0.8, mix=8),
        # Trees of up to 32 drafted tokens that are certain, float32 logits.
        dict(name="verify_trees", kind="verify", seqs=16, rows=33, ragged=True, shape="tree", vocab=157184,
             dtype="f32", temperature=1.0, mix=9),
    ]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_HEADS = [(4, 4, 64), (16, 16, 64), (16, 4, 64), (16, 4, 128), (32, 8, 128)]      # heads, K/V heads, head length


def draw(rng):
    kind = rng.choice(["norm", "train", "put", "shared", "shared", "verify", "verify"])
    heads, kv, hd = rng.choice(_HEADS)
    page = rng.choice([16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    mix = rng.randrange(1 << 30)
    if kind in ("norm", "train"):
        scaling = rng.choice(["none", "linear", "ntk", "yarn"])
        factor = 1.0 if scaling == "none" else round(rng.uniform(1.5, 16.0), 2)
        dtype = rng.choice(["bf16", "f16", "f32"])
        return dict(kind=kind, rows=_logint(rng, 1, 16384 * 20 // (heads + kv) if dtype != "f32" else 8192), heads=heads,
                    kv=kv, hd=hd, rot=rng.choice([hd, hd, hd // 2, 2 * rng.randint(2, hd // 2)]),
                    layout=rng.choice(["half", "interleaved"]), scaling=scaling, factor=factor, original=4096,
                    theta=rng.choice([10000.0, 500000.0]), dtype=dtype, gain=rng.choice([dtype, "f32"]),
                    far=_logint(rng, 64, 1 << 20))
    if kind == "put":
        return dict(kind=kind, seqs=_logint(rng, 1, 32), rows=_logint(rng, 1, 512), heads=heads, kv=kv, hd=hd,
                    page=page, len_lo=0, len_hi=_logint(rng, 1, 2048), dtype=dtype, src=rng.choice([dtype, "f32"]),
                    gain="f32", mix=mix)
    if kind == "shared":
        groups = _logint(rng, 1, 8)
        members = _logint(rng, 1, 64 // groups)
        mask = rng.choice(["full", "full", "tree"])
        hi = _logint(rng, 1, 32768 // groups)
        return dict(kind=kind, layers=rng.choice([1, 1, 2, 4]), groups=groups, members=members,
                    alone=rng.choice([0, 0, rng.randint(1, 4)]),
                    rows=_logint(rng, 1, max(1, min(40, 256 // (groups * members)))), ragged=rng.random() < 0.5, mask=mask,
                    heads=heads, kv=kv, hd=hd, page=page, prefix_lo=max(1, hi // rng.choice([1, 2, 8])), prefix_hi=hi,
                    tail_lo=0, tail_hi=_logint(rng, 1, 1024), dtype=dtype, mix=mix)
    shape = rng.choice(["chain", "tree"])
    vocab = _logint(rng, 100, 157184)
    rows = _logint(rng, 1, 48)
    return dict(kind=kind, seqs=_logint(rng, 1, max(1, min(64, (16 * 33 * 157184) // (2 * rows * vocab)))), rows=rows,
                ragged=rng.random() < 0.6, shape=shape, vocab=vocab, dtype=rng.choice(["bf16", "f16", "f32"]),
                temperature=rng.choice([1.0, 1.0, 0.7, 1.3]), mix=mix)


# ------------------------------------------------------------------ shape of a case

def _pages(n, page):
    return (n + page - 1) // page


def _plan(case):
    """Lengths, rows and groups of a case: what its user's program knows on the host."""
    rng = random.Random(case["mix"])
    top = case["rows"]
    if case["kind"] == "shared":
        group = [g for g in range(case["groups"]) for _ in range(case["members"])] + [-1] * case["alone"]
        rng.shuffle(group)
        B = len(group)
        prefix = [_logint(rng, case["prefix_lo"], case["prefix_hi"]) for _ in range(case["groups"])]
        tail = [rng.randint(case["tail_lo"], case["tail_hi"]) for _ in range(B)]
        first = [prefix[g] if g >= 0 else rng.choice(prefix) for g in group]
        lens = [a + b for a, b in zip(first, tail)]
        whole = [prefix[g] // case["page"] if g >= 0 else 0 for g in group]      # pages shared
        rows = [rng.randint(1, top) if case["ragged"] else top for _ in range(B)]
        return dict(lens=lens, rows=rows, group=group, whole=whole)
    B = case["seqs"]
    if case["kind"] == "put":
        lens = [_logint(rng, max(1, case["len_lo"]), max(1, case["len_hi"])) if case["len_hi"] else 0 for _ in range(B)]
        rows = [max(1, rng.randint(top // 4, top)) if top > 1 else 1 for _ in range(B)]
        return dict(lens=lens, rows=rows, group=[-1] * B, whole=[0] * B)
    rows = [rng.randint(1, top) if case["ragged"] else top for _ in range(B)]
    if case["ragged"] and B > 3:
        rows[rng.randrange(B)] = 0                    # a sequence that sits the pass out
    parent = []
    for n in rows:
        if case["shape"] == "chain":
            parent += [i - 1 for i in range(n)]
        else:
            parent += [-1 if i == 0 else rng.randrange(max(0, i - 6), i) for i in range(n)]
    return dict(rows=rows, parent=parent)


def _geometry(case):
    """(entries of a table row, pages of the pool) of a case."""
    p = _plan(case)
    need = [_pages(n + r, case["page"]) for n, r in zip(p["lens"], p["rows"])]
    own_pages = sum(n - w for n, w in zip(need, p["whole"]))
    shared = {g: w for g, w in zip(p["group"], p["whole"]) if g >= 0}
    return max(need), own_pages + sum(shared.values()) + 3


# ------------------------------------------------------------------ inputs

def _device():
    return torch.device("cuda")


def _generator(seed):
    g = torch.Generator(device=_device())
    g.manual_seed(int(seed))
    return g


def _randn(g, shape, dtype, scale=1.0):
    out = torch.empty(shape, dtype=dtype, device=_device())
    flat, step = out.view(-1), 1 << 26
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        flat[i:i + n] = (scale * torch.randn(n, generator=g, device=_device())).to(dtype)
    return out


def _starts(rows):
    out = [0]
    for n in rows:
        out.append(out[-1] + n)
    return out


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=_device())


def _tree(rows, seed):
    """Boolean lists [rows][rows] of one sequence: a drafted token sees its ancestors and itself."""
    rng = random.Random(seed)
    see = [[False] * rows for _ in range(rows)]
    for i in range(rows):
        if i and rng.random() < 0.98:
            see[i] = list(see[rng.randrange(max(0, i - 12), i)])
        see[i][i] = True
    return see


def _mask_words(case, plan, seed):
    """int32 [rows, words]: bit j of a row's words tells whether it sees row j of its sequence."""
    words = (case["rows"] + 31) // 32
    out = []
    for b, n in enumerate(plan["rows"]):
        for line in _tree(n, seed * 1009 + b):
            v = [0] * words
            for j, s in enumerate(line):
                if s:
                    v[j // 32] |= 1 << (j % 32)
            out.append([w - (1 << 32) if w >> 31 else w for w in v])
    return _ints(out)


def _meta(case, plan, seed):
    """[references | lengths | tables]: pages in a shuffled order, those of a group's prefix in all its tables."""
    width, n_pages = _geometry(case)
    order = list(range(n_pages))
    random.Random(seed).shuffle(order)
    order = iter(order)
    B = len(plan["rows"])
    ref, table, front = [0] * n_pages, [[-1] * width for _ in range(B)], {}
    for b in range(B):
        g = plan["group"][b]
        if g >= 0 and g not in front:
            front[g] = [next(order) for _ in range(plan["whole"][b])]
        pages = list(front.get(g, []))
        pages += [next(order) for _ in range(_pages(plan["lens"][b] + plan["rows"][b], case["page"]) - len(pages))]
        table[b][:len(pages)] = pages
        for p in pages:
            ref[p] += 1
    return _ints(ref + plan["lens"] + [t for row in table for t in row])


def _rope_args(case):
    if case["kind"] == "put":
        return dict(rot=case["hd"], layout="half", scaling="none", factor=1.0, original=0, theta=10000.0)
    return case


def _split_rows(g, T, case, dtype, scale=1.0):
    """Queries, keys and values of T rows, as one product gives them."""
    heads, kv, hd = case["heads"], case["kv"], case["hd"]
    qkv = _randn(g, (T, (heads + 2 * kv) * hd), dtype, scale)
    a, b = heads * hd, (heads + kv) * hd
    return qkv[:, :a].view(T, heads, hd), qkv[:, a:b].view(T, kv, hd), qkv[:, b:].view(T, kv, hd)


def _gains(g, case):
    dt = DTYPES[case["gain"]]
    return [(1.0 + 0.2 * torch.randn(case["hd"], generator=g, device=_device())).to(dt) for _ in range(2)]


def _verify_inputs(case, seed):
    g, plan = _generator(seed), _plan(case)
    T, V, dt = sum(plan["rows"]), case["vocab"], DTYPES[case["dtype"]]
    dev = _device()
    target = _randn(g, (T, V), dt, 2.0)
    n_top = min(8, V)
    # What the model thinks of holds most of the weight: tokens that differ within a row.
    top = torch.randint(0, V, (T, 1), generator=g, device=dev)
    top = (top + torch.arange(n_top, device=dev) * (V // n_top)) % V
    high = 12.0 + 6.0 * torch.rand(T, n_top, generator=g, device=dev)
    target.scatter_(1, top, high.to(dt))
    st = dict(plan=plan, target=target, row_start=_ints(_starts(plan["rows"])), draft=None)
    source = target
    if case["shape"] == "chain":
        st["draft"] = torch.empty_like(target)
        for i in range(T):
            st["draft"][i] = (target[i].float() + 0.7 * torch.randn(V, generator=g, device=dev)).to(dt)
        source = st["draft"]
    starts = _starts(plan["rows"])
    drawn = torch.zeros(T, dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(plan["rows"]):
        for i in range(n):
            p = plan["parent"][at]
            if i:                                     # drawn from what its parent's row says
                noise = -torch.log(-torch.log(torch.rand(V, generator=g, device=dev).clamp(1e-9, 1.0 - 1e-7)))
                drawn[at] = (source[starts[b] + p].float() / case["temperature"] + noise).argmax()
            at += 1
    st["tokens"] = drawn
    st["parent"] = _ints(plan["parent"]) if case["shape"] == "tree" else None
    st["u"] = torch.rand(T, generator=g, device=dev)
    st["u_next"] = torch.rand(len(plan["rows"]), generator=g, device=dev)
    return st


def _inputs(case, seed):
    """Tensors of a case, from the seed alone."""
    g, dev = _generator(seed), _device()
    if case["kind"] == "verify":
        return _verify_inputs(case, seed)
    if case["kind"] in ("norm", "train"):
        q, k, _ = _split_rows(g, case["rows"], case, DTYPES[case["dtype"]], 1.5)
        qg, kg = _gains(g, case)
        st = dict(q=q, k=k, q_gain=qg, k_gain=kg,
                  pos=torch.randint(0, case["far"], (case["rows"],), generator=g, device=dev, dtype=torch.int32))
        if case["kind"] == "train":
            st["dq"] = _randn(g, q.shape, q.dtype, 0.1)
            st["dk"] = _randn(g, k.shape, k.dtype, 0.1)
        return st
    plan = _plan(case)
    width, n_pages = _geometry(case)
    B, T = len(plan["rows"]), sum(plan["rows"])
    dt = DTYPES[case["dtype"]]
    st = dict(plan=plan, B=B, n_pages=n_pages, width=width, meta0=_meta(case, plan, seed),
              row_start=_ints(_starts(plan["rows"])))
    pool = (case.get("layers", 1), n_pages, case["kv"], case["page"], case["hd"])
    if case["kind"] == "put":
        st["k"], st["v"] = torch.zeros(pool, dtype=dt, device=dev), torch.zeros(pool, dtype=dt, device=dev)
        st["q_in"], st["k_in"], st["v_in"] = _split_rows(g, T, case, DTYPES[case["src"]], 1.5)
        st["q_gain"], st["k_gain"] = _gains(g, case)
        st["pos"] = _ints([n + i for n, r in zip(plan["lens"], plan["rows"]) for i in range(r)])
        return st
    st["k"], st["v"] = _randn(g, pool, dt), _randn(g, pool, dt)
    st["q"] = _randn(g, (case["layers"], T, case["heads"], case["hd"]), dt, 1.5)
    st["mask"] = None if case["mask"] == "full" else _mask_words(case, plan, seed)
    st["group"] = _ints(plan["group"])
    st["max_keys"] = max(n + r for n, r in zip(plan["lens"], plan["rows"]))
    by_group = [sum(r for r, x in zip(plan["rows"], plan["group"]) if x == y) for y in range(case["groups"])]
    st["max_group_rows"] = max(by_group)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    kind = case["kind"]
    if own and kind in ("norm", "train", "put"):
        from paper_2608_02625_amd import Rope

        r = _rope_args(case)
        st["rope"] = Rope(case["hd"], rot_dim=r["rot"], theta=r["theta"], interleaved=r["layout"] == "interleaved",
                          scaling=None if r["scaling"] == "none" else r["scaling"], factor=r["factor"],
                          original_len=r["original"])
    if own and kind in ("put", "shared"):
        from paper_2608_02625_amd import PagedCache

        c = PagedCache(case.get("layers", 1), st["n_pages"], case["page"], case["kv"], case["hd"], st["B"], st["width"],
                       dtype=DTYPES[case["dtype"]], device=_device(), k=st["k"], v=st["v"])
        c.meta.copy_(st["meta0"])
        st["cache"] = c
    if kind == "norm":
        st["out"] = torch.empty(st["q"].shape, dtype=st["q"].dtype, device=_device())
        st["k_out"] = torch.empty(st["k"].shape, dtype=st["k"].dtype, device=_device())
    if kind == "put":
        st["q_out"] = torch.empty(st["q_in"].shape, dtype=DTYPES[case["dtype"]], device=_device())
    if kind == "shared":
        st["out"] = torch.empty_like(st["q"])
    if "meta0" in st:
        n, b = st["n_pages"], st["B"]
        st["len"] = st["meta0"][n:n + b]
        st["table"] = st["meta0"][n + b:].view(b, st["width"])
    return st


# ------------------------------------------------------------------ one pass

def run(st):
    kind = st["case"]["kind"]
    return (_RUN_OWN if own else _RUN_PLAIN)[kind](st)


def _own_norm(st):
    q, k = st["rope"].norm_apply(st["q"], st["k"], st["pos"], st["q_gain"], st["k_gain"], eps=EPS, out=st["out"],
                                 k_out=st["k_out"])
    return {"q": q, "k": k}


def _own_train(st):
    leaves = [st[n].detach().requires_grad_() for n in ("q", "k", "q_gain", "k_gain")]
    q, k = st["rope"].norm_apply(leaves[0], leaves[1], st["pos"], leaves[2], leaves[3], eps=EPS)
    dq, dk, dqg, dkg = torch.autograd.grad((q, k), leaves, (st["dq"], st["dk"]))
    return {"q": q.detach(), "k": k.detach(), "dq": dq, "dk": dk, "dq_gain": dqg, "dk_gain": dkg}


def _own_put(st):
    q = st["cache"].append(0, st["k_in"], st["v_in"], st["row_start"], st["case"]["rows"], q=st["q_in"],
                           rope=st["rope"], positions=st["pos"], q_out=st["q_out"], q_gain=st["q_gain"],
                           k_gain=st["k_gain"], norm_eps=EPS)
    return {"q": q, "k": st["k"], "v": st["v"]}


def _own_shared(st):
    c, case = st["cache"], st["case"]
    share = c.share(st["row_start"], st["group"], st["q"].shape[1], case["rows"], st["max_group_rows"])
    for layer in range(case["layers"]):
        c.attend(layer, st["q"][layer], st["row_start"], case["rows"], mask=st["mask"], max_keys=st["max_keys"],
                 out=st["out"][layer], share=share)
    return st["out"]


def _own_verify(st):
    from paper_2608_02625_amd import verify

    case = st["case"]
    v = verify(st["row_start"], st["tokens"], st["target"], st["u"], st["u_next"], parent=st["parent"],
               draft=st["draft"], temperature=case["temperature"], max_rows=case["rows"])
    return {"next": v.next, "keep": v.keep, "keep_start": v.keep_start}


_RUN_OWN = dict(norm=_own_norm, train=_own_train, put=_own_put, shared=_own_shared, verify=_own_verify)


# ------------------------------------------------------------------ plain forms

def _frequencies(r, dev):
    """Angle per position of every pair, float64, and the factor on the rotated values."""
    i = torch.arange(r["rot"] // 2, dtype=torch.float64, device=dev)
    theta, s = r["theta"], r["factor"]
    if r["scaling"] == "ntk":
        theta = theta * s ** (r["rot"] / (r["rot"] - 2))
    f = theta ** (-2.0 * i / r["rot"])
    if r["scaling"] == "linear":
        f = f / s
    if r["scaling"] == "yarn":
        turns = r["original"] * f / (2.0 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / s
        return f, 0.1 * math.log(s) + 1.0
    return f, 1.0


def _rotate(x, pos, r, back=False):
    f, amp = _frequencies(r, x.device)
    ang = pos.double()[:, None] * f[None, :]
    cos = (amp * torch.cos(ang)).float()[:, None, :]
    sin = (amp * torch.sin(ang)).float()[:, None, :]
    if back:
        sin = -sin
    half, rot = r["rot"] // 2, r["rot"]
    y = x.clone()
    if r["layout"] == "half":
        a, b = x[..., :half], x[..., half:rot]
        y[..., :half] = a * cos - b * sin
        y[..., half:rot] = b * cos + a * sin
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2] = a * cos - b * sin
        y[..., 1:rot:2] = b * cos + a * sin
    return y


def _normed(x):
    """x over the root of its mean square, and one over that root."""
    x = x.float()
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r


def _plain_norm(st):
    for x, gain, out in (("q", "q_gain", "out"), ("k", "k_gain", "k_out")):
        st[out].copy_(_rotate(_normed(st[x])[0] * st[gain].float(), st["pos"], st["case"]))
    return {"q": st["out"], "k": st["k_out"]}


def _plain_train(st):
    out = {}
    for x in ("q", "k"):
        gain = st[x + "_gain"].float()
        n, r = _normed(st[x])
        out[x] = _rotate(n * gain, st["pos"], st["case"]).to(st[x].dtype)
        u = _rotate(st["d" + x].float(), st["pos"], st["case"], back=True)
        out[f"d{x}_gain"] = (u * n).sum((0, 1), dtype=torch.float64).to(st[x + "_gain"].dtype)
        h = u * gain
        out["d" + x] = (r * (h - n * (h * n).mean(-1, keepdim=True))).to(st[x].dtype)
    return out


def _plain_put(st):
    case = st["case"]
    t = torch.arange(st["k_in"].shape[0], device=st["row_start"].device)
    seq = torch.searchsorted(st["row_start"][1:].long(), t, right=True)
    at = st["len"][seq].long() + t - st["row_start"][seq].long()
    page, at = st["table"][seq, at // case["page"]].long(), at % case["page"]
    r = _rope_args(case)
    st["q_out"].copy_(_rotate(_normed(st["q_in"])[0] * st["q_gain"].float(), st["pos"], r))
    st["k"][0][page, :, at] = _rotate(_normed(st["k_in"])[0] * st["k_gain"].float(), st["pos"], r).to(st["k"].dtype)
    st["v"][0][page, :, at] = st["v_in"].to(st["v"].dtype)
    return {"q": st["q_out"], "k": st["k"], "v": st["v"]}


def _plain_shared(st):
    case, plan = st["case"], st["plan"]
    H, KV, hd, page = case["heads"], case["kv"], case["hd"], case["page"]
    bits = torch.arange(32, device=st["q"].device)
    for layer in range(case["layers"]):
        t0 = 0
        for b, n in enumerate(plan["rows"]):
            keys = plan["lens"][b] + n
            pages = st["table"][b, :_pages(keys, page)].long()
            k = st["k"][layer][pages].permute(1, 0, 2, 3).reshape(KV, -1, hd)[:, :keys].float()
            v = st["v"][layer][pages].permute(1, 0, 2, 3).reshape(KV, -1, hd)[:, :keys].float()
            q = st["q"][layer, t0:t0 + n].float().view(n, KV, H // KV, hd).permute(1, 2, 0, 3).reshape(KV, -1, hd)
            z = (torch.matmul(q, k.transpose(1, 2)) / math.sqrt(hd)).view(KV, H // KV, n, keys)
            if st["mask"] is not None:
                see = ((st["mask"][t0:t0 + n, :, None] >> bits) & 1).bool().reshape(n, -1)[:, :n]
                z[..., plan["lens"][b]:].masked_fill_(~see, -math.inf)
            z = torch.exp(z - z.amax(-1, keepdim=True))
            z = z / z.sum(-1, keepdim=True)
            o = torch.matmul(z.view(KV, -1, keys), v).view(KV, H // KV, n, hd).permute(2, 0, 1, 3)
            st["out"][layer, t0:t0 + n] = o.reshape(n, H, hd).to(st["out"].dtype)
            t0 += n
    return st["out"]


def _chances(z, temperature):
    z = z.double() / temperature
    z = torch.exp(z - z.amax(-1, keepdim=True))
    return z / z.sum(-1, keepdim=True)


def _plain_verify(st):
    case, starts = st["case"], st["row_start"].long()
    first, count = starts[:-1], starts[1:] - starts[:-1]
    T, B = st["tokens"].shape[0], count.shape[0]
    dev = starts.device
    p = _chances(st["target"], case["temperature"])
    q = None if st["draft"] is None else _chances(st["draft"], case["temperature"])
    seq = torch.searchsorted(starts[1:], torch.arange(T, device=dev), right=True)
    kept = torch.zeros(T + 1, dtype=torch.int64, device=dev)
    one = torch.arange(B, device=dev)
    root = first.clamp(max=T - 1)
    kept.index_put_((torch.where(count > 0, first, T),), torch.ones_like(first))
    left = p[root]                                    # what the node at hand has left to say
    at = torch.zeros_like(first)
    for i in range(1, case["rows"]):
        row = (first + i).clamp(max=T - 1)
        parent = torch.full_like(first, i - 1) if st["parent"] is None else st["parent"][row].long()
        here = (i < count) & (parent == at)
        x = st["tokens"][row].long()
        px = left[one, x]
        if q is None:
            good = here & (st["u"][row].double() * left.sum(-1) < px)
            left[one, x] = torch.where(here & ~good, torch.zeros_like(px), px)
        else:
            before = q[(first + at).clamp(max=T - 1)]
            good = here & (st["u"][row].double() * before[one, x] < px)
            rest = (left - before).clamp(min=0.0)
            left = torch.where((here & ~good & (rest.sum(-1) > 0))[:, None], rest, left)
        left = torch.where(good[:, None], p[row], left)
        at = torch.where(good, torch.full_like(at, i), at)
        kept.index_put_((torch.where(good, row, T),), torch.ones_like(row))
    c = left.cumsum(-1)
    token = (c <= (st["u_next"].double() * c[:, -1])[:, None]).sum(-1).clamp(max=case["vocab"] - 1)
    kept = kept[:T]
    place = torch.where(kept > 0, kept.cumsum(0) - 1, T)
    keep = torch.full((T + 1,), -1, dtype=torch.int32, device=dev)
    keep.index_put_((place,), (torch.arange(T, device=dev) - first[seq]).to(torch.int32))
    keep_start = torch.zeros(B + 1, dtype=torch.int32, device=dev)
    keep_start[1:] = torch.zeros(B, dtype=torch.int64, device=dev).index_add_(0, seq, kept).cumsum(0).to(torch.int32)
    return {"next": torch.where(count > 0, token, -1).to(torch.int32), "keep": keep[:T], "keep_start": keep_start}


_RUN_PLAIN = dict(norm=_plain_norm, train=_plain_train, put=_plain_put, shared=_plain_shared, verify=_plain_verify)


# ------------------------------------------------------------------ work

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] in ("norm", "train"):
        values = case["rows"] * (case["heads"] + case["kv"]) * case["hd"]
        gain = 2 * case["hd"] * (4 if case["gain"] == "f32" else 2)
        if case["kind"] == "norm":
            return {"bytes": 2 * values * size + gain + 4 * case["rows"], "flops": 8 * values}
        return {"bytes": 4 * values * size + 2 * gain + 4 * case["rows"], "flops": 24 * values}
    plan = _plan(case)
    T = sum(plan["rows"])
    if case["kind"] == "verify":
        logits = T * case["vocab"] * (2 if case["shape"] == "chain" else 1)
        return {"bytes": logits * size + 16 * T, "flops": 2 * logits}
    hd, kv, heads = case["hd"], case["kv"], case["heads"]
    if case["kind"] == "put":
        src = 4 if case["src"] == "f32" else 2
        values = T * (heads + 2 * kv) * hd
        return {"bytes": values * (src + size) + 4 * T, "flops": 8 * values}
    shared = {g: w * case["page"] for g, w in zip(plan["group"], plan["whole"]) if g >= 0}
    keys = sum(shared.values())
    pairs = 0
    for n, r, w in zip(plan["lens"], plan["rows"], plan["whole"]):
        keys += n + r - w * case["page"]
        pairs += n * r + (r * r if case["mask"] == "full" else 6 * r)
    mask = 0 if case["mask"] == "full" else 4 * T * ((case["rows"] + 31) // 32)
    return {"bytes": case["layers"] * (2 * keys * kv * hd * size + 2 * T * heads * hd * size + mask),
            "flops": case["layers"] * 4 * pairs * heads * hd}


# ------------------------------------------------------------------ float64 reference

def _turns64(r, pos):
    """e^(i angle) of every (row, pair) in float64, with the factor on them."""
    f = []
    for i in range(r["rot"] // 2):
        base = r["theta"]
        if r["scaling"] == "ntk":
            base *= math.pow(r["factor"], r["rot"] / (r["rot"] - 2.0))
        w = math.exp(-(2.0 * i / r["rot"]) * math.log(base))
        if r["scaling"] == "linear":
            w /= r["factor"]
        elif r["scaling"] == "yarn":                  # wavelengths shorter than original/32 stay, longer than it stretch
            per = r["original"] * w / (2.0 * math.pi)
            g = min(1.0, max(0.0, (per - 1.0) / (32.0 - 1.0)))
            w = (1.0 - g) * (w / r["factor"]) + g * w
        f.append(w)
    amp = 1.0 + 0.1 * math.log(r["factor"]) if r["scaling"] == "yarn" else 1.0
    ang = torch.outer(pos.double(), torch.tensor(f, dtype=torch.float64, device=pos.device))
    return torch.complex(amp * ang.cos(), amp * ang.sin())


def _rows64(x, gain, turns, r):
    """Normalised and rotated rows in float64; differentiable."""
    y = x * torch.rsqrt(x.square().mean(-1, True) + EPS) * gain
    n = r["rot"] // 2
    if r["layout"] == "half":
        z = torch.complex(y[..., :n], y[..., n:2 * n]) * turns[:, None, :]
        front = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.complex(y[..., 0:2 * n:2], y[..., 1:2 * n:2]) * turns[:, None, :]
        front = torch.stack([z.real, z.imag], -1).flatten(-2)
    return torch.cat([front, y[..., 2 * n:]], -1)


def _exact_verify(case, st):
    """One sequence after the other, as the rule reads."""
    plan, V = st["plan"], case["vocab"]
    starts = _starts(plan["rows"])
    tokens, u, u_next = st["tokens"].tolist(), st["u"].double().tolist(), st["u_next"].double().tolist()
    nxt, keep, keep_start = [], [], [0]

    def says(z):
        return torch.softmax(z.double() / case["temperature"], -1)

    for b, n in enumerate(plan["rows"]):
        at, path = 0, [0] if n else []
        token = -1
        if n:
            p = says(st["target"][starts[b]])
            for i in range(1, n):
                r = starts[b] + i
                if plan["parent"][r] != at:
                    continue
                x = tokens[r]
                if st["draft"] is None:
                    if u[r] * p.sum().item() < p[x].item():
                        at, p = i, says(st["target"][r])
                        path.append(i)
                    else:
                        p[x] = 0.0
                    continue
                q = says(st["draft"][starts[b] + at])
                if u[r] * q[x].item() < p[x].item():
                    at, p = i, says(st["target"][r])
                    path.append(i)
                    continue
                rest = torch.relu(p - q)
                if rest.sum().item() > 0:
                    p = rest
                break
            c = p.cpu().cumsum(0)
            token = min(V - 1, int(torch.searchsorted(c, u_next[b] * c[-1], right=True)))
        nxt.append(token)
        keep += path
        keep_start.append(len(keep))
    keep += [-1] * (starts[-1] - len(keep))
    return {"next": _ints(nxt), "keep": _ints(keep), "keep_start": _ints(keep_start)}


def exact(case, seed):
    st = _inputs(case, seed)
    kind = case["kind"]
    if kind == "verify":
        return _exact_verify(case, st)
    if kind in ("norm", "train"):
        turns = _turns64(case, st["pos"])
        out = {}
        for x in ("q", "k"):
            a, g = st[x].double(), st[x + "_gain"].double()
            if kind == "train":
                a.requires_grad_()
                g.requires_grad_()
            y = _rows64(a, g, turns, case)
            out[x] = y.detach()
            if kind == "train":
                out["d" + x], out[f"d{x}_gain"] = torch.autograd.grad(y, (a, g), st["d" + x].double())
        return out
    plan, page = st["plan"], case["page"]
    B, P, width = st["B"], st["n_pages"], st["width"]
    meta = st["meta0"].tolist()
    lens = meta[P:P + B]
    table = [meta[P + B + b * width:P + B + (b + 1) * width] for b in range(B)]
    if kind == "put":
        r = _rope_args(case)
        turns = _turns64(r, st["pos"])
        q = _rows64(st["q_in"].double(), st["q_gain"].double(), turns, r)
        k = _rows64(st["k_in"].double(), st["k_gain"].double(), turns, r)
        v = st["v_in"].double()
        K, V = st["k"].double(), st["v"].double()
        page_of = [table[b][(lens[b] + i) // page] for b in range(B) for i in range(plan["rows"][b])]
        place = [(lens[b] + i) % page for b in range(B) for i in range(plan["rows"][b])]
        page_of, place = torch.tensor(page_of, device=K.device), torch.tensor(place, device=K.device)
        K[0].permute(0, 2, 1, 3)[page_of, place] = k
        V[0].permute(0, 2, 1, 3)[page_of, place] = v
        return {"q": q, "k": K, "v": V}
    H, KV, hd = case["heads"], case["kv"], case["hd"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["q"].device)
    t = 0
    for b, n in enumerate(plan["rows"]):
        keys = lens[b] + n
        ids = torch.tensor(table[b][:_pages(keys, page)], device=st["q"].device)
        see = None
        if st["mask"] is not None:
            see = torch.ones(n, keys, dtype=torch.bool, device=st["q"].device)
            see[:, lens[b]:] = torch.tensor(_tree(n, seed * 1009 + b), device=st["q"].device)
        for layer in range(case["layers"]):
            for h in range(KV):
                K = st["k"][layer, ids, h].reshape(-1, hd)[:keys].double()
                V = st["v"][layer, ids, h].reshape(-1, hd)[:keys].double()
                for j in range(h * (H // KV), (h + 1) * (H // KV)):
                    z = st["q"][layer, t:t + n, j].double() @ K.T * hd ** -0.5
                    if see is not None:
                        z = z.masked_fill(~see, -math.inf)
                    out[layer, t:t + n, j] = torch.softmax(z, -1) @ V
        t += n
    return out
