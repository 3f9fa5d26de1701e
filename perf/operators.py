"""The operators of a paged K/V cache, as cases that can be timed and compared.

  append   tsd_append_paged_kv: the position rotation of new query and key rows, keys and values into their pages
  token    tsd_paged_attention: one new token per sequence over its pages
  verify   VerifyStep.attention_paged: a verification pass's attention layer, the cached keys read from pages

A page holds `page` consecutive tokens of one sequence; key t of sequence s is row t % page of page table[s, t // page].  The cache is in the
model's type or in 8-bit codes (e4m3) with one scale per kv head.  What no sequence uses holds NaN in the attention cases, and table entries
behind a sequence's last page are -1, as a pool that has just been allocated leaves them.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
FP8 = torch.float8_e4m3fn


# ------------------------------------------------------------------------------------------ cases
def _append(name, S, n, Hq, Hkv, d, page, dtype, cache, start, **more):
    """n rows per sequence behind a cache of about `start` tokens.  blocks > 1: the rows are one block of `blocks` per sequence, rotated before.
    rot: how many of the d dimensions turn; pairs: "half" (j, j + rot / 2) or "next" (2j, 2j + 1)."""
    c = dict(kind="append", S=S, n=n, Hq=Hq, Hkv=Hkv, d=d, page=page, dtype=dtype, cache=cache, start=start, blocks=1, rot=d, pairs="half",
             ragged=False)
    c.update(more)
    return dict(c, name=name) if name else c


def _token(name, S, cap, Hq, Hkv, d, page, dtype, cache, ragged):
    c = dict(kind="token", S=S, cap=cap, Hq=Hq, Hkv=Hkv, d=d, page=page, dtype=dtype, cache=cache, ragged=ragged)
    return dict(c, name=name) if name else c


def _verify(name, S, B, R, cap, Hq, Hkv, d, page, dtype, cache, ragged):
    c = dict(kind="verify", S=S, B=B, R=R, cap=cap, Hq=Hq, Hkv=Hkv, d=d, page=page, dtype=dtype, cache=cache, ragged=ragged)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One new token for each of eight requests: the call made once per layer and token, where latency counts.
        _append("append_one_token", 8, 1, 32, 32, 128, 64, "bf16", "bf16", 736, ragged=True),
        # The prompts of a batch go into the cache: 16 sequences of 1504 tokens, rotated queries for the attention that follows.
        _append("append_prompts", 16, 1504, 32, 32, 128, 64, "bf16", "bf16", 0),
        # A chunk of a long context: requests of different lengths, far positions, grouped heads, neighbouring pairs, 8-bit pages of 16 tokens.
        _append("append_far_e4m3", 6, 701, 28, 4, 128, 16, "bf16", "e4m3", 120000, pairs="next", ragged=True),
        # The accepted node's block of 32 rows out of 32 nodes, already rotated, behind the cache of each of 16 requests.
        _append("append_accepted", 16, 32, 32, 8, 64, 32, "bf16", "bf16", 1472, blocks=32, rot=0, ragged=True),
        # One request's next token over a short context, as many key heads as query heads: latency.
        _token("token_one_request", 1, 768, 32, 32, 128, 64, "bf16", "bf16", False),
        # A server's batch: 48 requests of 0 to 4096 tokens, seven query heads to a key head, small pages.
        _token("token_batch_ragged", 48, 4096, 28, 4, 128, 16, "bf16", "bf16", True),
        # Two requests with long documents.
        _token("token_long", 2, 131072, 28, 4, 128, 64, "bf16", "bf16", False),
        # A large batch whose cache is kept in 8 bits.
        _token("token_batch_e4m3", 64, 1504, 32, 32, 128, 32, "bf16", "e4m3", True),
        # fp32 with 64-wide heads, as a user checks a model with: the smallest attention.
        _token("token_fp32_head64", 3, 256, 4, 4, 64, 32, "f32", "f32", True),
        # One request's verification pass: an 8-node tree over 736 cached tokens.
        _verify("verify_one_request", 1, 8, 32, 736, 32, 32, 128, 32, "bf16", "bf16", False),
        # Long contexts of different lengths with full 32-node trees and grouped heads: the largest.
        _verify("verify_long_gqa", 4, 32, 32, 5056, 28, 4, 128, 64, "bf16", "bf16", True),
        # Trees cut to an odd 13 nodes, 64-wide heads, the cache in 8 bits.
        _verify("verify_e4m3_head64", 4, 13, 32, 1200, 32, 8, 64, 16, "bf16", "e4m3", True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_any(rng):
    kind = rng.choice(["append", "append", "token", "token", "token", "verify", "verify"])
    group = rng.choice([1, 1, 2, 4, 7, 8])
    Hkv = rng.choice([1, 2, 4, 8]) if group > 1 else rng.choice([4, 16, 32])
    d = rng.choice([64, 128, 128])
    page = rng.choice([8, 16, 16, 32, 64, 64, 128])
    dtype, cache = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "e4m3"), ("bf16", "e4m3"), ("f32", "f32")])
    ragged = rng.random() < 0.6
    if kind == "append":
        blocks = rng.choice([1, 1, 1, rng.randint(2, 32)])
        n = rng.choice([1, _log_int(rng, 2, 2048)]) if blocks == 1 else 32
        rot = 0 if blocks > 1 else rng.choice([d, d, d // 2, 16, 0])
        return _append(None, _log_int(rng, 1, 48), n, Hkv * group, Hkv, d, page, dtype, cache, rng.choice([0, _log_int(rng, 1, 8192), 120000]),
                       blocks=blocks, rot=rot, pairs=rng.choice(["half", "half", "next"]), ragged=ragged)
    if kind == "token":
        return _token(None, _log_int(rng, 1, 64), _log_int(rng, 1, 131072), Hkv * group, Hkv, d, page, dtype, cache, ragged)
    if dtype == "f32":  # the fp32 path serves checking, at checking's sizes
        return _verify(None, rng.choice([1, 2]), rng.randint(1, 8), 32, _log_int(rng, 8, 768), Hkv * group, Hkv, d, page, dtype, cache, ragged)
    return _verify(None, _log_int(rng, 1, 8), _log_int(rng, 1, 32), rng.choice([32, 32, 64]), _log_int(rng, 8, 5056), Hkv * group, Hkv, d, page,
                   dtype, cache, ragged)


def draw(rng):
    """1 to 48 sequences of 1 to 2048 new rows; caches of 1 to 131072 tokens for 1 to 64 sequences; trees of 1 to 32 nodes over 8 to 5056
    tokens; key heads that 1 to 8 query heads share; never more than the largest listed case of the kind."""
    largest = {}
    for c in listed():
        w = work(c)
        for key in ("bytes", "flops"):
            largest[c["kind"], key] = max(largest.get((c["kind"], key), 0), w[key])
    while True:
        case = _draw_any(rng)
        w = work(case)
        room = 0.1 if case["dtype"] == "f32" and case["kind"] == "verify" else 1.0
        if all(w[key] <= room * largest[case["kind"], key] for key in ("bytes", "flops")):
            return case


# ----------------------------------------------------------------------------------------- inputs
def _spread(count, most, least, ragged):
    """`count` lengths of at most `most`: all the same, or spread down to `least`, the smallest ones among them."""
    if not ragged:
        return [most] * count
    lens = [most - (7919 * i) % (most - least + 1) for i in range(count)]
    if count > 2:
        lens[1], lens[2] = least, min(most, least + 1)
    return lens


def _capacity(case):
    rows = case["start"] + case["n"] if case["kind"] == "append" else case["cap"]
    return -(-rows // case["page"]) * case["page"]


def _lens(case):
    """Cached tokens per sequence: before the call for an append, what the attention reads otherwise."""
    if case["kind"] == "append":
        return _spread(case["S"], case["start"], case["start"] * 7 // 8, case["ragged"])
    if case["kind"] == "token":
        return _spread(case["S"], case["cap"], 0, case["ragged"])
    return _spread(case["S"], case["cap"], case["cap"] // 2, case["ragged"])


def _new_rows(case):
    return _spread(case["S"], case["n"], 0, case["ragged"] and case["blocks"] == 1 and case["n"] > 1)


def _pages(case, gen, used):
    """Pools and table.  `used[s] = (first, last)`: the tokens whose pages sequence s has been given."""
    S, page, Hkv, d = case["S"], case["page"], case["Hkv"], case["d"]
    per_seq = _capacity(case) // page
    owned = torch.zeros((S, per_seq), dtype=torch.bool)
    for s, (first, last) in enumerate(used):
        if last > first:
            owned[s, first // page : (last - 1) // page + 1] = True
    n_pages = int(owned.sum()) + 3
    order = torch.randperm(n_pages, generator=gen, device=DEV, dtype=torch.int64)[: n_pages - 3].to(torch.int32)
    table = torch.full((S, per_seq), -1, dtype=torch.int32, device=DEV)
    table[owned.to(DEV)] = order
    shape = (n_pages, page, Hkv, d)
    st = dict(table=table)
    for name in ("k", "v"):
        x = torch.randn(shape, generator=gen, device=DEV)
        if case["cache"] == "e4m3":
            scale = (4.0 + torch.rand(Hkv, generator=gen, device=DEV)) / 448.0
            st[name + "_scale"] = scale
            st[name + "_pages"] = (x / scale[:, None]).clamp_(-448, 448).to(FP8)
        else:
            st[name + "_scale"] = None
            st[name + "_pages"] = x.to(DTYPES[case["dtype"]])
    return st


def _poison(case, st, lens):
    """NaN in every row of the pools that no sequence uses."""
    page = case["page"]
    live = torch.zeros(st["k_pages"].shape[:2], dtype=torch.bool, device=DEV)
    t = torch.arange(_capacity(case), device=DEV)
    for s, n in enumerate(lens):
        rows = t[:n]
        live[st["table"][s, rows // page].long(), rows % page] = True
    for name in ("k_pages", "v_pages"):
        pool = st[name].view(torch.uint8) if case["cache"] == "e4m3" else st[name]
        pool.masked_fill_(~live[:, :, None, None], 0x7F if case["cache"] == "e4m3" else math.nan)


def _prepare_append(case, gen):
    S, n, blocks, Hq, Hkv, d = (case[x] for x in ("S", "n", "blocks", "Hq", "Hkv", "d"))
    dt = DTYPES[case["dtype"]]
    lens, new = _lens(case), _new_rows(case)
    st = _pages(case, gen, [(a, a + n) for a in lens])
    rnd = lambda heads: torch.randn((S, blocks * n, heads, d), generator=gen, device=DEV).to(dt)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    st.update(k=rnd(Hkv), v=rnd(Hkv), q=rnd(Hq) if blocks == 1 else None, first_slot=ints(lens), n_new=ints(new) if case["ragged"] else None,
              block=torch.randint(0, blocks, (S,), generator=gen, device=DEV, dtype=torch.int32) if blocks > 1 else None,
              inv_freq=1e4 ** (-torch.arange(0, case["rot"], 2, device=DEV, dtype=torch.float32) / case["rot"]) if case["rot"] else None)
    st["q_out"] = torch.zeros_like(st["q"]) if blocks == 1 else None
    if own:
        from paper_2608_27514_b200 import binding as B

        st["handle"] = B.make_paged_cache(st["k_pages"], st["v_pages"], st["table"], st["k_scale"], st["v_scale"])
        st["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return st


def _prepare_token(case, gen):
    S, Hq, d = case["S"], case["Hq"], case["d"]
    dt = DTYPES[case["dtype"]]
    lens = _lens(case)
    st = _pages(case, gen, [(0, n) for n in lens])
    _poison(case, st, lens)
    st.update(q=torch.randn((S, Hq, d), generator=gen, device=DEV).to(dt), lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
              sm_scale=d**-0.5, out=torch.empty((S, Hq, d), dtype=dt, device=DEV), lse=torch.empty((S, Hq), dtype=torch.float32, device=DEV))
    if own:
        from paper_2608_27514_b200 import binding as B

        st["handle"] = B.make_paged_cache(st["k_pages"], st["v_pages"], st["table"], st["k_scale"], st["v_scale"])
        st["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        st["workspace"] = torch.zeros(max(16, B.tsd_paged_attention_workspace_bytes(st["handle"], Hq)), dtype=torch.uint8, device=DEV)
    return st


def _prepare_verify(case, gen):
    S, B, R, Hq, Hkv, d = (case[x] for x in ("S", "B", "R", "Hq", "Hkv", "d"))
    dt = DTYPES[case["dtype"]]
    lens = _lens(case)
    st = _pages(case, gen, [(0, n) for n in lens])
    _poison(case, st, lens)
    rnd = lambda heads: torch.randn((S, B * R, heads, d), generator=gen, device=DEV).to(dt)
    st.update(q=rnd(Hq), k_draft=rnd(Hkv), v_draft=rnd(Hkv), lens=torch.tensor(lens, dtype=torch.int32, device=DEV), sm_scale=d**-0.5)
    if own:
        from paper_2608_27514_b200 import binding as Bind
        from paper_2608_27514_b200.step import VerifyStep

        st["handle"] = Bind.make_paged_cache(st["k_pages"], st["v_pages"], st["table"], st["k_scale"], st["v_scale"])
        st["step"] = VerifyStep(S, B, R, case["cap"], Hq, Hkv, d, 64, 1, dt, DEV)
        st["step"].build_mask(None, st["lens"])
    return st


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(9000 + int(seed) % (1 << 30))
    make = {"append": _prepare_append, "token": _prepare_token, "verify": _prepare_verify}[case["kind"]]
    return dict(make(case, gen), case=dict(case))


# ------------------------------------------------------------------------------------- plain forms
def _rotated(x, angle, rot, pairs):
    """x [S, n, H, d] turned by angle [S, n, rot / 2], in 32 bits."""
    x = x.float()
    if not rot:
        return x
    c, s = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    turn, rest = x[..., :rot], x[..., rot:]
    a, b = (turn[..., : rot // 2], turn[..., rot // 2 :]) if pairs == "half" else (turn[..., 0::2], turn[..., 1::2])
    a, b = a * c - b * s, a * s + b * c
    turn = torch.cat([a, b], -1) if pairs == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([turn, rest], -1)


def _plain_append(st):
    case = st["case"]
    S, n, page, rot = case["S"], case["n"], case["page"], case["rot"]
    i = torch.arange(n, device=DEV)
    slot = st["first_slot"][:, None].long() + i
    k, v = st["k"], st["v"]
    if st["block"] is not None:
        rows = (st["block"][:, None].long() * n + i)[:, :, None, None].expand(-1, -1, *k.shape[2:])
        k, v = k.gather(1, rows), v.gather(1, rows)
    angle = slot[:, :, None].double() * st["inv_freq"].double() if rot else None
    valid = (i < (st["n_new"][:, None] if st["n_new"] is not None else n)).expand(S, n)
    at = st["table"].gather(1, slot // page).long(), slot % page
    for name, x in (("k", _rotated(k, angle, rot, case["pairs"])), ("v", v.float())):
        pool = st[name + "_pages"]
        if case["cache"] == "e4m3":
            codes = (x / st[name + "_scale"][:, None]).clamp(-448, 448).to(FP8).view(torch.uint8)
            raw = pool.view(torch.uint8)
            raw[at] = torch.where(valid[:, :, None, None], codes, raw[at])
        else:
            pool[at] = torch.where(valid[:, :, None, None], x.to(pool.dtype), pool[at])
    out = dict(k_pages=st["k_pages"], v_pages=st["v_pages"])
    if st["q"] is not None:
        q = _rotated(st["q"], angle, rot, case["pairs"]).to(st["q"].dtype)
        st["q_out"].copy_(torch.where(valid[:, :, None, None], q, st["q_out"]))
        out["q_out"] = st["q_out"]
    return out


def _dense(st, name):
    """The pages in the order of the keys, in 32 bits: [S, capacity, Hkv, d], 0 where no sequence uses them."""
    pool, at = st[name + "_pages"], st["table"].clamp(min=0).long()
    x = (pool.view(torch.uint8)[at].view(FP8) if st["case"]["cache"] == "e4m3" else pool[at]).flatten(1, 2).float()
    if st[name + "_scale"] is not None:
        x = x * st[name + "_scale"][:, None]
        if st["case"]["kind"] == "verify":  # the verification pass reads an 8-bit cache as bf16 values
            x = x.bfloat16().float()
    live = torch.arange(x.shape[1], device=DEV) < st["lens"][:, None]
    return torch.where(live[:, :, None, None], x, 0.0), live


def _weights(scores, seen):
    """Softmax over the last axis where `seen`, its log-sum-exp; rows that see nothing: 0 and -inf."""
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = (scores - top).exp()
    total = w.sum(-1, keepdim=True)
    return w / total.clamp(min=1e-30), (total.log() + top).squeeze(-1)


def _plain_token(st):
    case = st["case"]
    S, Hkv, d = case["S"], case["Hkv"], case["d"]
    k, live = _dense(st, "k")
    q = st["q"].float().view(S, Hkv, -1, d)
    w, lse = _weights(torch.einsum("shgd,sthd->shgt", q, k) * st["sm_scale"], live[:, None, None])
    del k
    v, _ = _dense(st, "v")
    out = torch.einsum("shgt,sthd->shgd", w, v)
    return dict(out=out.flatten(1, 2).to(st["q"].dtype), lse=lse.flatten(1, 2))


def _plain_verify(st):
    case = st["case"]
    S, Hkv, d, N, R = case["S"], case["Hkv"], case["d"], case["B"] * case["R"], case["R"]
    k, live = _dense(st, "k")
    v, _ = _dense(st, "v")
    k, v = torch.cat([k, st["k_draft"].float()], 1), torch.cat([v, st["v_draft"].float()], 1)
    branch = torch.arange(N, device=DEV) // R
    same = branch[:, None] == branch
    seen = torch.cat([live[:, None].expand(-1, N, -1), same.expand(S, -1, -1)], 2)
    q = st["q"].float().view(S, N, Hkv, -1, d)
    w, lse = _weights(torch.einsum("snhgd,sthd->shgnt", q, k) * st["sm_scale"], seen[:, None, None])
    out = torch.einsum("shgnt,sthd->snhgd", w, v)
    return dict(out=out.flatten(2, 3).to(st["q"].dtype), lse=lse.flatten(1, 2))


# ------------------------------------------------------------------------------------------ passes
def _own_append(st):
    from paper_2608_27514_b200 import binding as B

    case = st["case"]
    B.tsd_append_paged_kv(st["handle"], st["k"], st["v"], st["first_slot"], st["n_new"], inv_freq=st["inv_freq"],
                          interleaved=case["pairs"] == "next", q=st["q"], q_out=st["q_out"], block=st["block"], n_rows=case["n"],
                          status=st["status"])
    out = dict(k_pages=st["k_pages"], v_pages=st["v_pages"])
    if st["q"] is not None:
        out["q_out"] = st["q_out"]
    return out


def _own_token(st):
    from paper_2608_27514_b200 import binding as B

    B.tsd_paged_attention(st["handle"], st["q"], st["lens"], st["out"], st["lse"], st["sm_scale"], st["workspace"], st["status"])
    return dict(out=st["out"], lse=st["lse"])


def _own_verify(st):
    step = st["step"]
    out = step.attention_paged(st["q"], st["handle"], st["k_draft"], st["v_draft"], st["sm_scale"])
    return dict(out=out, lse=step.attn_lse)


def run(state):
    if own:
        return {"append": _own_append, "token": _own_token, "verify": _own_verify}[state["case"]["kind"]](state)
    return {"append": _plain_append, "token": _plain_token, "verify": _plain_verify}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------- exact
def _exact_append(case, st):
    """Row by row from the definition: every new row's slot is looked up, its rotation taken as a complex product."""
    n, page, rot = case["n"], case["page"], case["rot"]
    count = st["n_new"].tolist() if st["n_new"] is not None else [n] * case["S"]
    res = {name: st[name].double() for name in ("k_pages", "v_pages")}
    if st["q"] is not None:
        res["q_out"] = st["q_out"].double()

    def turned(x, pos):
        x = x.double()
        if not rot:
            return x
        z = x[..., :rot].reshape(*x.shape[:-1], *((2, rot // 2) if case["pairs"] == "half" else (rot // 2, 2)))
        z = z.transpose(-1, -2) if case["pairs"] == "half" else z
        phase = pos.double()[:, None, None] * st["inv_freq"].double()
        z = torch.view_as_complex(z.contiguous()) * torch.polar(torch.ones_like(phase), phase)
        z = torch.view_as_real(z)
        z = z.transpose(-1, -2) if case["pairs"] == "half" else z
        return torch.cat([z.reshape(*x.shape[:-1], rot), x[..., rot:]], -1)

    for s in range(case["S"]):
        m, at = count[s], int(st["first_slot"][s])
        if m == 0:
            continue
        r0 = int(st["block"][s]) * n if st["block"] is not None else 0
        pos = torch.arange(at, at + m, device=DEV)
        pages, rows = st["table"][s].long()[pos // page], pos % page
        k, v = turned(st["k"][s, r0 : r0 + m], pos), st["v"][s, r0 : r0 + m].double()
        if case["cache"] == "e4m3":
            k, v = (k / st["k_scale"].double()[:, None]).clamp(-448, 448), (v / st["v_scale"].double()[:, None]).clamp(-448, 448)
        res["k_pages"][pages, rows], res["v_pages"][pages, rows] = k, v
        if st["q"] is not None:
            res["q_out"][s, :m] = turned(st["q"][s, :m], pos)
    return res


def _keys_of(case, st, s):
    """The cached keys and values of one sequence in 64 bits: [Hkv, len, d] each."""
    t = torch.arange(int(st["lens"][s]), device=DEV)
    pages, rows = st["table"][s].long()[t // case["page"]], t % case["page"]
    both = []
    for name in ("k", "v"):
        pool = st[name + "_pages"]
        if case["cache"] == "e4m3":
            x = pool.view(torch.uint8)[pages, rows].view(FP8).double() * st[name + "_scale"].double()[:, None]
        else:
            x = pool[pages, rows].double()
        both.append(x.transpose(0, 1))
    return both


def _exact_token(case, st):
    Hkv, group, d = case["Hkv"], case["Hq"] // case["Hkv"], case["d"]
    outs, lses = [], []
    for s in range(case["S"]):
        k, v = _keys_of(case, st, s)
        q = st["q"][s].double().view(Hkv, group, d)
        if k.shape[1] == 0:
            outs.append(torch.zeros_like(q).flatten(0, 1))
            lses.append(torch.full((case["Hq"],), -math.inf, dtype=torch.float64, device=DEV))
            continue
        a = q @ k.mT * st["sm_scale"]
        outs.append((torch.softmax(a, -1) @ v).flatten(0, 1))
        lses.append(torch.logsumexp(a, -1).flatten())
    return dict(out=torch.stack(outs), lse=torch.stack(lses))


def _exact_verify(case, st):
    B, R, Hkv, group, d = case["B"], case["R"], case["Hkv"], case["Hq"] // case["Hkv"], case["d"]
    outs, lses = [], []
    for s in range(case["S"]):
        k, v = _keys_of(case, st, s)
        if case["cache"] == "e4m3":  # the verification pass reads an 8-bit cache as bf16 values
            k, v = k.float().bfloat16().double(), v.float().bfloat16().double()
        q = st["q"][s].double().view(B, R, Hkv, group, d).permute(0, 2, 3, 1, 4)  # [B, Hkv, group, R, d]
        kd, vd = (st[x][s].double().view(B, R, Hkv, 1, d).permute(0, 2, 3, 1, 4) for x in ("k_draft", "v_draft"))
        cached, mine = q @ k[None, :, None].mT * st["sm_scale"], q @ kd.mT * st["sm_scale"]
        total = torch.logaddexp(torch.logsumexp(cached, -1), torch.logsumexp(mine, -1))
        out = (cached - total[..., None]).exp() @ v[None, :, None] + (mine - total[..., None]).exp() @ vd
        outs.append(out.permute(0, 3, 1, 2, 4).reshape(B * R, Hkv * group, d))
        lses.append(total.permute(1, 2, 0, 3).reshape(Hkv * group, B * R))
    return dict(out=torch.stack(outs), lse=torch.stack(lses))


def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "token": _exact_token, "verify": _exact_verify}[case["kind"]](case, st)


# -------------------------------------------------------------------------------------- accounting
def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    cached = 1 if case["cache"] == "e4m3" else size
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    if case["kind"] == "append":
        rows = sum(_new_rows(case))
        q = 2 * Hq * d * size if case["blocks"] == 1 else 0
        return dict(bytes=float(rows * (q + 2 * Hkv * d * (size + cached))), flops=float(rows * 3 * case["rot"] * (Hkv + (Hq if q else 0))))
    keys = sum(_lens(case))
    if case["kind"] == "token":
        return dict(bytes=float(2 * keys * Hkv * d * cached + case["S"] * Hq * (2 * d * size + 4)), flops=4.0 * keys * Hq * d)
    S, N = case["S"], case["B"] * case["R"]
    nbytes = 2 * keys * Hkv * d * cached + S * N * (2 * Hq * d + 2 * Hkv * d) * size + 4 * S * N * Hq
    return dict(bytes=float(nbytes), flops=4.0 * d * Hq * N * (keys + S * case["R"]))
