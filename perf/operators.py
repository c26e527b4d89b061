"""Performance cases of the latent-attention and page operators: attention over a paged cache that holds one latent
vector a token (decode step in absorbed form, prompts in expanded form), the append that fills such a cache, and the
copies that forking, compacting and joining branches make of a cache's pages.

A case names its operator in `op` and holds the sizes; block tables, lengths and values are drawn from it and the seed.
A latent page is [(latent_dim + rope_dim) / 8][16 tokens][8]; a K tile of the KV pool is [d / 8][16][8], a V tile
[16 / 4][d][4].  Pages of a sequence are scattered over the pool, as an engine that has been running leaves them.
"""
import math

import numpy as np
import torch

own = False

PAGE, ROPE = 16, 64
DEVICE = "cuda:0"

# --------------------------------------------------------------------------- cases
ATTENTION = dict(
    heads=16, latent=512, hd=128,  # query heads on this GPU, latent width, width of a head's keys (without the rotated part) and values
    serial=0, ctx_lo=0, ctx_hi=0,  # requests of one sequence: count, context range
    parallel=0, pre_lo=0, pre_hi=0, width_lo=0, width_hi=0, suf_lo=0, suf_hi=0,  # requests of several branches on a shared prefix
    lens=0,                        # seed of the lengths
    lse=False,
)
PROMPT = dict(ATTENTION, new_lo=0, new_hi=0)  # new tokens of each sequence; the rest of its context is cached already
APPEND = dict(latent=512, tokens=0, holes=False)  # holes: a padded batch, some of whose rows hold no token
PAGES = dict(kind="kv", hkv=8, d=128, latent=512, layers=1)


def _case(op, name=None, **kw):
    base = dict(decode=ATTENTION, prompt=PROMPT, append=APPEND, copy=dict(PAGES, moves=0),
                pack=dict(PAGES, requests=0, pre_lo=0, pre_hi=0, width_lo=0, width_hi=0, suf_lo=0, suf_hi=0, lens=0))[op]
    c = dict(op=op, **dict(base, **kw))
    return c if name is None else dict(name=name, **c)


# the benchmark's batches: serial requests beside requests with 4 to 8 branches; long shared documents
MIXED = dict(serial=16, ctx_lo=1024, ctx_hi=4096, parallel=8, pre_lo=2048, pre_hi=8192, width_lo=4, width_hi=8,
             suf_lo=0, suf_hi=1024, lens=20260503)


def listed():
    return [
        # one user, one request on one rank of a tensor-parallel group of eight: interactive latency
        _case("decode", "decode_one", heads=16, serial=1, ctx_lo=701, ctx_hi=701, lens=1),
        # the serial batch on such a rank: streaming the cache is all there is
        _case("decode", "decode_serial", heads=16, serial=32, ctx_lo=1024, ctx_hi=4096, lens=20260502),
        # the mixed batch with all heads of a model on one GPU (data-parallel attention): a row of the cache meets 128 heads
        _case("decode", "decode_mixed", heads=128, lse=True, **MIXED),
        # long shared documents, 16 branches each
        _case("decode", "decode_long_prefix", heads=64, serial=32, ctx_lo=1024, ctx_hi=8192, parallel=8, pre_lo=32768,
              pre_hi=32768, width_lo=16, width_hi=16, suf_lo=0, suf_hi=2048, lens=20260504),
        # a short question to a small model
        _case("prompt", "prompt_one", heads=16, latent=256, hd=64, serial=1, ctx_lo=131, ctx_hi=131, new_lo=131, new_hi=131, lens=2),
        # ragged prompts, nothing cached, some of a few tokens
        _case("prompt", "prompt_ragged", heads=32, serial=12, ctx_lo=5, ctx_hi=4096, new_lo=1 << 30, new_hi=1 << 30, lens=25, lse=True),
        # chunks of long prompts beside branches' headers behind a shared prefix, all heads on one GPU
        _case("prompt", "prompt_chunk", heads=128, serial=2, ctx_lo=16384, ctx_hi=32768, parallel=2, pre_lo=2048, pre_hi=8192,
              width_lo=4, width_hi=8, suf_lo=24, suf_hi=300, new_lo=1024, new_hi=1024, lens=11),
        # the tokens of a decode step
        _case("append", "append_step", tokens=60),
        # the tokens of a batch of prompts, padded
        _case("append", "append_prompt", tokens=16384, holes=True),
        # branches that fork in the middle of a page: each gets a copy of the last one, in every layer
        _case("copy", "copy_fork", layers=8, moves=7),
        # the live pages of a pool moved to its front
        _case("copy", "copy_compact", layers=4, moves=4096),
        # joined branches become one contiguous prefix of the next phase of their request
        _case("pack", "pack_join", kind="kv", layers=4, requests=8, pre_lo=2048, pre_hi=8192, width_lo=4, width_hi=8, suf_lo=1,
              suf_hi=1024, lens=20260503),
    ]


MOST_FLOPS, MOST_BYTES = 3.0e12, 4 << 30  # of a drawn case: no more than the largest listed ones


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["decode", "decode", "prompt", "prompt", "append", "copy", "pack"])
        c = _case(op)
        if op in ("decode", "prompt"):
            latent, hd = rng.choice([(512, 128), (512, 128), (256, 64), (256, 128), (512, 64)])
            c.update(heads=rng.choice([1, 5, 8, 16, 20, 32, 64, 128, 128]), latent=latent, hd=hd, lens=rng.randrange(1 << 30),
                     lse=rng.random() < 0.5)
            branches = rng.random() < 0.6
            if not branches or rng.random() < 0.7:
                lo = log_int(1, 8192)
                c.update(serial=log_int(1, 128 if op == "decode" else 24), ctx_lo=lo, ctx_hi=min(32768, log_int(lo, 4 * lo)))
            if branches:
                lo, suf, w = log_int(1, 16384), log_int(1, 2048), log_int(2, 40 if op == "decode" else 8)
                c.update(parallel=log_int(1, 16 if op == "decode" else 4), pre_lo=lo, pre_hi=min(32768, log_int(lo, 4 * lo)),
                         width_lo=w, width_hi=w + rng.randrange(0, 5), suf_lo=rng.choice([0, suf // 2]), suf_hi=suf)
            if op == "prompt":
                n = log_int(1, 4096)
                c.update(new_lo=rng.choice([0, 1, n // 2]), new_hi=n)
                if sum(n for _, seqs in _requests(c) for _, n in seqs) == 0:
                    continue
        elif op == "append":
            c.update(latent=rng.choice([256, 512, 512]), tokens=log_int(1, 16384), holes=rng.random() < 0.5)
        else:
            c.update(kind=rng.choice(["kv", "latent"]), hkv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128]),
                     latent=rng.choice([256, 512]), layers=rng.randint(1, 12))
            if op == "copy":
                c.update(moves=log_int(1, 4096))
            else:
                lo, suf, w = log_int(1, 8192), log_int(1, 2048), log_int(1, 17)
                c.update(requests=log_int(1, 12), pre_lo=lo, pre_hi=log_int(lo, 4 * lo), width_lo=w, width_hi=w + rng.randrange(0, 3),
                         suf_lo=rng.choice([0, 1, suf // 2]), suf_hi=suf, lens=rng.randrange(1 << 30))
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= (MOST_BYTES if op in ("copy", "pack") else MOST_BYTES / 8):
            return c


# --------------------------------------------------------------------------- integers of a batch
def _some(r, lo, hi, n):
    return [int(x) for x in (r.integers(lo, hi, size=n, endpoint=True) if lo < hi else np.full(n, lo))]


def _requests(case):
    """[(prefix tokens, [(private tokens, new tokens), ...]), ...]; of a decode step every sequence has one query row."""
    r = np.random.Generator(np.random.PCG64(case["lens"]))
    ctx = _some(r, case["ctx_lo"], case["ctx_hi"], case["serial"])
    pre = _some(r, case["pre_lo"], case["pre_hi"], case["parallel"])
    wid = _some(r, case["width_lo"], case["width_hi"], case["parallel"])
    reqs = [(0, [c]) for c in ctx]
    reqs += [(p, _some(r, case["suf_lo"], case["suf_hi"], w)) for p, w in zip(pre, wid)]
    out = []
    for p, suf in reqs:
        if case["op"] == "prompt":
            new = [min(n, s) for n, s in zip(_some(r, case["new_lo"], case["new_hi"], len(suf)), suf)]
        else:
            new = [1] * len(suf)
        out.append((p, list(zip(suf, new))))
    return out


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _scatter(seed, used):
    """A pool with 10 % to spare and its pages in random order."""
    n = max(1, math.ceil(1.1 * used))
    return n, np.random.Generator(np.random.PCG64(seed)).permutation(n).astype(np.int32)


def _batch(case, seed):
    reqs = _requests(case)
    used = sum(_pages(p) + sum(_pages(s) for s, _ in seqs) for p, seqs in reqs)
    n_pages, free = _scatter(seed, used)
    cur, rows, group, prefix, suffix, new = 0, [], [], [], [], []
    for g, (p, seqs) in enumerate(reqs):
        shared = free[cur:cur + _pages(p)]
        cur += len(shared)
        for s, n in seqs:
            rows.append(np.concatenate([shared, free[cur:cur + _pages(s)]]))
            cur += _pages(s)
            group.append(g)
            prefix.append(p)
            suffix.append(s)
            new.append(n)
    table = np.full((len(rows), max(1, max(len(x) for x in rows))), -1, np.int32)
    for s, row in enumerate(rows):
        table[s, :len(row)] = row
    i32 = lambda v: np.array(v, np.int32)  # noqa: E731
    return dict(table=table, group=i32(group), prefix=i32(prefix), suffix=i32(suffix), new=i32(new), n_pages=n_pages)


def _join(case, seed):
    """Requests whose branches have ended: source rows (prefix, then each branch's pages), and where their tokens go.  Full pages of
    the prefix stay where they are (first_token); the rest is written to new pages."""
    r = np.random.Generator(np.random.PCG64(case["lens"]))
    pre = _some(r, case["pre_lo"], case["pre_hi"], case["requests"])
    wid = _some(r, case["width_lo"], case["width_hi"], case["requests"])
    suf = [_some(r, case["suf_lo"], case["suf_hi"], w) for w in wid]
    first = [p // PAGE * PAGE for p in pre]
    n_src = [_pages(p) + sum(_pages(x) for x in s) for p, s in zip(pre, suf)]
    n_dst = [_pages(p + sum(s) - f) for p, s, f in zip(pre, suf, first)]
    n_pages, free = _scatter(seed, sum(n_src) + sum(n_dst))
    cut = np.cumsum([0] + n_src + n_dst)
    table = np.full((len(pre), max(1, max(n_src))), -1, np.int32)
    dst = np.full((len(pre), max(1, max(n_dst))), -1, np.int32)
    for i, (a, b) in enumerate(zip(n_src, n_dst)):
        table[i, :a] = free[cut[i]:cut[i] + a]
        dst[i, :b] = free[cut[len(pre) + i]:cut[len(pre) + i] + b]
    i32 = lambda v: np.array(v, np.int32)  # noqa: E731
    return dict(table=table, prefix=i32(pre), seg_start=i32(np.cumsum([0] + [len(s) for s in suf])),
                seg_len=i32([x for s in suf for x in s]), first=i32(first), dst=dst, n_pages=n_pages)


# --------------------------------------------------------------------------- inputs
def _normal(gen, *shape, std=1.0):
    return torch.empty(shape, device=DEVICE, dtype=torch.bfloat16).normal_(0.0, std, generator=gen)


def _pool_shape(case, n):
    if case["kind"] == "kv":
        return (n, 2, case["hkv"], PAGE * case["d"])
    return (n, (case["latent"] + ROPE) // 8, PAGE, 8)


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed + 1000)
    op = case["op"]
    if op in ("decode", "prompt"):
        b = _batch(case, seed)
        H, R, hd = case["heads"], case["latent"], case["hd"]
        # latents of unit scale (they come out of a norm), weights that keep that scale in the expanded keys and values
        return dict(batch=b, q=_normal(gen, int(b["new"].sum()), H, hd + ROPE), w=_normal(gen, H, 2 * hd, R, std=R ** -0.5),
                    pages=_normal(gen, b["n_pages"], (R + ROPE) // 8, PAGE, 8))
    if op == "append":
        n, R = case["tokens"], case["latent"]
        n_pages, free = _scatter(seed, _pages(n))
        slots = (free[np.arange(n) // PAGE].astype(np.int64) * PAGE + np.arange(n) % PAGE)
        if case["holes"]:  # rows behind a prompt's end
            slots[np.random.Generator(np.random.PCG64(seed + 1)).random(n) < 0.2] = -1
        return dict(n_pages=n_pages, slots=torch.from_numpy(slots).to(DEVICE), latent=_normal(gen, n, R), rope=_normal(gen, n, ROPE),
                    pages=_normal(gen, n_pages, (R + ROPE) // 8, PAGE, 8))
    if op == "copy":
        n_pages, free = _scatter(seed, 2 * case["moves"])
        b = dict(n_pages=n_pages, src=free[:case["moves"]].copy(), dst=free[case["moves"]:2 * case["moves"]].copy())
    else:
        b = _join(case, seed)
    return dict(batch=b, pools=[_normal(gen, *_pool_shape(case, b["n_pages"])) for _ in range(case["layers"])])


_kept = {}


def _kept_once(key, make):
    """Contexts live as long as the process, as an engine has them."""
    if key not in _kept:
        _kept[key] = make()
    return _kept[key]


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    op = case["op"]
    if op in ("decode", "prompt"):
        b, H = s["batch"], case["heads"]
        n = s["q"].shape[0]
        s["out"] = torch.empty(n, H, case["hd"], device=DEVICE, dtype=torch.bfloat16)
        s["lse"] = torch.empty(n, H, device=DEVICE) if case["lse"] else None
        if own:
            from paper_2605_06914_amd import LatentContext
            s["ctx"] = _kept_once(("latent", H, case["latent"], case["hd"]), lambda: LatentContext(H, case["latent"], case["hd"], device=0))
            args = (b["table"], b["group"], b["prefix"], b["suffix"])
            if op == "decode":  # one plan serves all layers of a step: a layer's call finds it built
                s["plan"] = s["ctx"].plan_build(*args, b["n_pages"])
            else:
                s["plan"] = s["ctx"].prompt_plan_build(*args, b["new"], b["n_pages"])
    elif op == "append":
        if own:
            from paper_2605_06914_amd import LatentContext
            s["ctx"] = _kept_once(("latent", 16, case["latent"], 128), lambda: LatentContext(16, case["latent"], 128, device=0))
    elif own:
        from paper_2605_06914_amd import PageMover
        key = (case["kind"], case["hkv"], case["d"]) if case["kind"] == "kv" else (case["kind"], case["latent"])
        s["mover"] = _kept_once(key, lambda: PageMover.kv(case["hkv"], case["d"], device=0) if case["kind"] == "kv" else PageMover.latent(case["latent"], device=0))
    return s


# --------------------------------------------------------------------------- one pass
def run(state):
    op = state["case"]["op"]
    if not own:
        return dict(decode=_plain_decode, prompt=_plain_prompt, append=_plain_append, copy=_plain_copy, pack=_plain_pack)[op](state)
    b = state.get("batch")
    if op == "decode":
        state["ctx"].decode_step_attention(state["plan"], state["q"], state["w"], state["pages"], state["out"], state["lse"])
        return {"out": state["out"], "lse": state["lse"]}
    if op == "prompt":
        state["ctx"].prompt_attention(state["plan"], state["q"], state["w"], state["pages"], state["out"], state["lse"])
        return {"out": state["out"], "lse": state["lse"]}
    if op == "append":
        state["ctx"].append(state["latent"], state["rope"], state["slots"], state["pages"], state["n_pages"])
        return {"pages": state["pages"]}
    if op == "copy":
        state["mover"].copy(state["pools"], b["src"], b["dst"], b["n_pages"])
    else:
        state["mover"].pack(state["pools"], b["table"], b["prefix"], b["seg_start"], b["seg_len"], b["dst"], b["n_pages"], first_token=b["first"])
    return {"pools": state["pools"]}


# --------------------------------------------------------------------------- plain forms
def _tokens(pages, ids, n):
    """The first n tokens of latent pages `ids`, [n, latent + rope], in 32 bits."""
    t = pages[torch.from_numpy(ids.astype(np.int64)).to(pages.device)]
    return t.permute(0, 2, 1, 3).reshape(len(ids) * PAGE, 8 * pages.shape[1])[:n].float()


def _softmax_parts(score):
    m = score.amax(-1, keepdim=True)
    p = torch.exp(score - m)
    l = p.sum(-1, keepdim=True)
    return p / l, (m + torch.log(l)).squeeze(-1)


def _plain_decode(s):
    """Absorbed: the key weights go into the query, the value weights come behind the sum over tokens."""
    case, b = s["case"], s["batch"]
    H, R, hd = case["heads"], case["latent"], case["hd"]
    w = s["w"].float()
    q = s["q"].float()
    q_lat = torch.matmul(q[:, :, :hd].transpose(0, 1), w[:, :hd]).transpose(0, 1)  # [S, H, R]
    q_all = torch.cat([q_lat, q[:, :, hd:]], -1)
    o_lat = torch.empty_like(q_lat)
    lse = torch.empty(q.shape[0], H, device=q.device)
    shared = (-1, None)
    for i in range(q.shape[0]):
        p, n = int(b["prefix"][i]), int(b["suffix"][i])
        if shared[0] != b["group"][i]:
            shared = (b["group"][i], _tokens(s["pages"], b["table"][i, :_pages(p)], p))
        c = torch.cat([shared[1], _tokens(s["pages"], b["table"][i, _pages(p):_pages(p) + _pages(n)], n)])
        prob, lse[i] = _softmax_parts(torch.matmul(q_all[i], c.t()) * (hd + ROPE) ** -0.5)
        o_lat[i] = torch.matmul(prob, c[:, :R])
    out = torch.matmul(o_lat.transpose(0, 1), w[:, hd:].transpose(1, 2)).transpose(0, 1)
    return {"out": out.to(torch.bfloat16).contiguous(), "lse": lse if case["lse"] else None}


def _plain_prompt(s):
    """Expanded: every head's keys and values of every token, then causal attention; some heads at a time."""
    case, b = s["case"], s["batch"]
    H, R, hd = case["heads"], case["latent"], case["hd"]
    w = s["w"].float()
    out = torch.empty(s["q"].shape[0], H, hd, device=DEVICE, dtype=torch.bfloat16)
    lse = torch.empty(s["q"].shape[0], H, device=DEVICE)
    r0 = 0
    for i in range(len(b["new"])):
        p, n, new = int(b["prefix"][i]), int(b["suffix"][i]), int(b["new"][i])
        if new == 0:
            continue
        c = torch.cat([_tokens(s["pages"], b["table"][i, :_pages(p)], p), _tokens(s["pages"], b["table"][i, _pages(p):_pages(p) + _pages(n)], n)])
        T = p + n
        ahead = torch.arange(T, device=DEVICE)[None, :] > torch.arange(T - new, T, device=DEVICE)[:, None]
        some = max(1, min(H, (1 << 28) // (new * T)))
        for h0 in range(0, H, some):
            wh = w[h0:h0 + some]
            k = torch.matmul(c[:, :R], wh[:, :hd].transpose(1, 2))
            v = torch.matmul(c[:, :R], wh[:, hd:].transpose(1, 2))
            q = s["q"][r0:r0 + new, h0:h0 + some].float().transpose(0, 1)
            score = torch.matmul(q[:, :, :hd], k.transpose(1, 2)) + torch.matmul(q[:, :, hd:], c[:, R:].t())
            score = (score * (hd + ROPE) ** -0.5).masked_fill_(ahead, -math.inf)
            prob, l = _softmax_parts(score)
            out[r0:r0 + new, h0:h0 + some] = torch.matmul(prob, v).transpose(0, 1).to(torch.bfloat16)
            lse[r0:r0 + new, h0:h0 + some] = l.t()
        r0 += new
    return {"out": out, "lse": lse if case["lse"] else None}


def _plain_append(s):
    keep = torch.nonzero(s["slots"] >= 0).squeeze(-1)
    slots = s["slots"][keep]
    rows = torch.cat([s["latent"], s["rope"]], -1)[keep]
    s["pages"][slots // PAGE, :, slots % PAGE] = rows.view(len(slots), -1, 8)
    return {"pages": s["pages"]}


def _plain_copy(s):
    src = torch.from_numpy(s["batch"]["src"].astype(np.int64)).to(DEVICE)
    dst = torch.from_numpy(s["batch"]["dst"].astype(np.int64)).to(DEVICE)
    for pool in s["pools"]:
        pool[dst] = pool[src]
    return {"pools": s["pools"]}


def _pack_slots(b):
    """(source slot, destination slot) of every token that moves."""
    src, dst = [], []
    for i in range(len(b["prefix"])):
        entry, slots = 0, []
        for n in [int(b["prefix"][i])] + [int(x) for x in b["seg_len"][b["seg_start"][i]:b["seg_start"][i + 1]]]:
            t = np.arange(n)
            slots.append(b["table"][i, entry + t // PAGE].astype(np.int64) * PAGE + t % PAGE)
            entry += _pages(n)
        slots = np.concatenate(slots)[int(b["first"][i]):]
        t = np.arange(len(slots))
        src.append(slots)
        dst.append(b["dst"][i, t // PAGE].astype(np.int64) * PAGE + t % PAGE)
    return np.concatenate(src), np.concatenate(dst)


def _plain_pack(s):
    case = s["case"]
    src, dst = (torch.from_numpy(x).to(DEVICE) for x in _pack_slots(s["batch"]))
    for pool in s["pools"]:
        if case["kind"] == "latent":
            pool[dst // PAGE, :, dst % PAGE] = pool[src // PAGE, :, src % PAGE]
        else:
            n, hkv, d = pool.shape[0], case["hkv"], case["d"]
            k = pool.view(n, 2, hkv, d // 8, PAGE, 8)
            k[dst // PAGE, 0, :, :, dst % PAGE] = k[src // PAGE, 0, :, :, src % PAGE]
            v = pool.view(n, 2, hkv, PAGE // 4, d, 4)
            v[dst // PAGE, 1, :, dst % PAGE // 4, :, dst % 4] = v[src // PAGE, 1, :, src % PAGE // 4, :, src % 4]
    return {"pools": s["pools"]}


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    """Attention: every visible token's latent once (a shared prefix once a request), queries, weights and results once; the products
    of the form that the operator takes.  Moves and appends: each moved token read once and written once."""
    op = case["op"]
    if op in ("decode", "prompt"):
        H, R, hd = case["heads"], case["latent"], case["hd"]
        reqs = [(p, [x for x in seqs if x[1]]) for p, seqs in _requests(case)]
        unique = sum((p if seqs else 0) + sum(s for s, _ in seqs) for p, seqs in reqs)
        rows = sum(n for _, seqs in reqs for _, n in seqs)
        nbytes = unique * (R + ROPE) * 2 + rows * H * (2 * hd + ROPE) * 2 + H * 2 * hd * R * 2 + (rows * H * 4 if case["lse"] else 0)
        if op == "decode":
            seen = sum(p + s for p, seqs in reqs for s, _ in seqs)
            return {"bytes": nbytes, "flops": H * (seen * 2 * (2 * R + ROPE) + rows * 4 * hd * R)}
        seen = sum(n * (p + s) - n * (n - 1) // 2 for p, seqs in reqs for s, n in seqs)
        return {"bytes": nbytes, "flops": H * (seen * 2 * (2 * hd + ROPE) + unique * 4 * hd * R)}
    if op == "append":
        return {"bytes": case["tokens"] * ((case["latent"] + ROPE) * 4 + 8), "flops": 0}
    token = 2 * (2 * case["hkv"] * case["d"] if case["kind"] == "kv" else case["latent"] + ROPE)
    if op == "copy":
        return {"bytes": 2 * case["layers"] * case["moves"] * PAGE * token, "flops": 0}
    b = _join(case, 0)
    return {"bytes": 2 * case["layers"] * token * int(b["prefix"].sum() + b["seg_len"].sum() - b["first"].sum()), "flops": 0}


# --------------------------------------------------------------------------- the same in 64 bits
def _exact_rows(pages, ids, n):
    """Tokens one page after the other, [n, latent + rope]."""
    rows = [pages[int(i)].double().transpose(0, 1).reshape(PAGE, -1) for i in ids]
    return torch.cat(rows)[:n] if rows else torch.zeros(0, pages.shape[1] * 8, device=pages.device, dtype=torch.float64)


def _exact_attention(case, s):
    """Row by row of the definition: head h's key of token t is (W_k[h] c_t, r_t), its value W_v[h] c_t; query i of a sequence's n
    new ones sees all but the last n - 1 - i tokens."""
    b, H, R, hd = s["batch"], case["heads"], case["latent"], case["hd"]
    w = s["w"].double()
    q = s["q"].double()
    out = torch.zeros(q.shape[0], H, hd, device=DEVICE, dtype=torch.float64)
    lse = torch.zeros(q.shape[0], H, device=DEVICE, dtype=torch.float64)
    r0 = np.concatenate([[0], np.cumsum(b["new"])])
    for g in range(int(b["group"][-1]) + 1):
        members = np.nonzero(b["group"] == g)[0]
        p = int(b["prefix"][members[0]])
        head_rows = _exact_rows(s["pages"], b["table"][members[0], :_pages(p)], p)
        tails = [_exact_rows(s["pages"], b["table"][i, _pages(p):_pages(p) + _pages(int(b["suffix"][i]))], int(b["suffix"][i])) for i in members]
        for h in range(H):
            def keys_values(c):
                return torch.cat([c[:, :R] @ w[h, :hd].T, c[:, R:]], 1), c[:, :R] @ w[h, hd:].T
            k0, v0 = keys_values(head_rows)
            for i, tail in zip(members, tails):
                n = int(b["new"][i])
                if n == 0:
                    continue
                k1, v1 = keys_values(tail)
                rows = slice(int(r0[i]), int(r0[i]) + n)
                sc = torch.cat([q[rows, h] @ k0.T, q[rows, h] @ k1.T], 1) / math.sqrt(hd + ROPE)
                T = p + int(b["suffix"][i])
                sc = torch.where(torch.ones(n, T, device=DEVICE, dtype=torch.bool).tril(T - n), sc, -math.inf)
                lse[rows, h] = torch.logsumexp(sc, 1)
                pr = torch.exp(sc - lse[rows, h][:, None])
                out[rows, h] = pr[:, :p] @ v0 + pr[:, p:] @ v1
    return {"out": out, "lse": lse if case["lse"] else None}


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op in ("decode", "prompt"):
        return _exact_attention(case, s)
    if op == "append":
        rows = torch.cat([s["latent"], s["rope"]], 1)
        t = s["pages"].permute(0, 2, 1, 3).reshape(s["n_pages"] * PAGE, -1)  # a row a slot
        keep = s["slots"] >= 0
        t[s["slots"][keep]] = rows[keep]
        return {"pages": t.view(s["n_pages"], PAGE, -1, 8).transpose(1, 2).contiguous()}
    b = s["batch"]
    done = []
    for pool in s["pools"]:
        if op == "copy":
            kept = pool.clone()
            for i, j in zip(b["src"], b["dst"]):
                kept[int(j)] = pool[int(i)]
        else:
            src, dst = (torch.from_numpy(x).to(DEVICE) for x in _pack_slots(b))
            if case["kind"] == "latent":
                t = pool.transpose(1, 2).reshape(-1, case["latent"] + ROPE)
                t[dst] = t[src]
                kept = t.view(pool.shape[0], PAGE, -1, 8).transpose(1, 2).contiguous()
            else:
                n, hkv, d = pool.shape[0], case["hkv"], case["d"]
                k = pool[:, 0].view(n, hkv, d // 8, PAGE, 8).permute(0, 3, 1, 2, 4).reshape(n * PAGE, -1)
                v = pool[:, 1].view(n, hkv, PAGE // 4, d, 4).permute(0, 2, 4, 1, 3).reshape(n * PAGE, -1)
                k[dst], v[dst] = k[src], v[src]
                k = k.view(n, PAGE, hkv, d // 8, 8).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1)
                v = v.view(n, PAGE // 4, 4, hkv, d).permute(0, 3, 1, 4, 2).reshape(n, hkv, -1)
                kept = torch.stack([k, v], 1)
        done.append(kept)
    return {"pools": done}
