"""The operators around drafted tokens and the paged 8-bit cache, as measurable cases.

Five calls, in the order in which a serving program with drafted tokens makes them: a tree of drafts becomes masks and
positions (`prepare`); the drafts attend to kept ranges of the fixed context, to the paged cache and to one another (`attend`, a prompt
behind a context among them: there the drafts are a chain); what the model agrees with is accepted (`accept`) and written into the cache in
8 bits (`commit`); a cache is read back in 16 bits (`read`).  Data are drawn on the GPU from the seed alone.
"""
import math
import random

import torch

own = False

D = 128
BLOCK = 64                                   # keys of the fixed context that share a scale
SM_SCALE = float(torch.tensor(1.0 / math.sqrt(D), dtype=torch.float32))
E_MIN, E_MAX = -64, 64                       # exponents of a block's scale
F8, F16, F32, F64, I32, I64, U8 = torch.float8_e4m3fn, torch.float16, torch.float32, torch.float64, torch.int32, torch.int64, torch.uint8


def _prepare(name, B, T, ragged=False):
    return dict(name=name, kind="prepare", B=B, T=T, ragged=ragged)


def _accept(name, B, T, ragged=False):
    return dict(name=name, kind="accept", B=B, T=T, ragged=ragged)


def _attend(name, B, H, G, T, tree, L, C, keep, user, page, ragged=False):
    """T drafts a sequence, a tree or a chain; keep: share of the fixed context's keys that a head keeps on average (C = 0: no
    fixed context); user: the longest sequence in the cache."""
    return dict(name=name, kind="attend", B=B, H=H, G=G, T=T, tree=tree, L=L, C=C, keep=keep, user=user, page=page, ragged=ragged)


def _commit(name, B, H, T, path, page, old):
    """path: the most drafts that a sequence accepts (0: all T rows in order, a prompt); old: the most tokens it has so far."""
    return dict(name=name, kind="commit", B=B, H=H, T=T, path=path, page=page, old=old)


def _read(name, B, H, U, page):
    return dict(name=name, kind="read", B=B, H=H, U=U, page=page)


def listed():
    return [
        # One sequence, a small tree: launch latency.
        _prepare("prepare_one", 1, 16),
        # A full batch of large trees of uneven size.
        _prepare("prepare_batch", 64, 256, True),
        # A small tree of few heads over a short context: launches and dependent reads.
        _attend("tree_4k", 1, 4, 1, 8, True, 4096, 64, 1 / 4, 128, 64),
        # One sequence's tree of 64 drafts, grouped heads, a 32K context.
        _attend("tree_32k", 1, 8, 4, 64, True, 32768, 1024, 1 / 8, 512, 64),
        # A batch with trees of uneven, odd size, and long answers behind a 128K context.
        _attend("tree_batch", 16, 8, 4, 13, True, 131072, 4096, 1 / 16, 4096, 16, True),
        # The next turn's prompt behind a 32K context and an answer of 1000 tokens: a chain, bound by the products.
        _attend("chain_2k", 1, 8, 4, 2048, False, 32768, 1024, 1 / 8, 1000, 64),
        # What the model agrees with, one sequence.
        _accept("accept_one", 1, 16),
        # The same of a large batch.
        _accept("accept_batch", 256, 64, True),
        # A few accepted drafts of every sequence of a batch.
        _commit("commit_drafts", 16, 8, 64, 6, 64, 2048),
        # Prompts of uneven length, normed and rotated already.
        _commit("commit_prompts", 4, 8, 8000, 0, 64, 700),
        # One answer read back.
        _read("read_answer", 1, 8, 500, 64),
        # Long conversations read back, to be clustered or to prefill behind them.
        _read("read_batch", 4, 32, 8192, 16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["prepare", "accept", "attend", "attend", "attend", "attend", "commit", "read"])
    ragged = rng.random() < 0.5
    if kind in ("prepare", "accept"):
        T = _log_int(rng, 1, 256)
        return dict(kind=kind, B=_log_int(rng, 1, 256 * 64 // T), T=T, ragged=ragged)
    H, G = rng.choice([(1, 8), (2, 16), (4, 1), (5, 3), (8, 4), (8, 5), (12, 1), (20, 1), (32, 1)])
    page = rng.choice([16, 32, 64])
    if kind == "commit":
        B = _log_int(rng, 1, 64)
        path = rng.choice([0, 1, _log_int(rng, 2, 20)])
        T = max(path, _log_int(rng, 1, 128 if path else 8000 * 32 // (B * H)))
        return dict(kind=kind, B=B, H=H, T=T, path=path, page=page, old=_log_int(rng, 1, 2000))
    if kind == "read":
        B = _log_int(rng, 1, 16)
        return dict(kind=kind, B=B, H=H, U=_log_int(rng, 1, min(32768, 8192 * 128 // (B * H))), page=page)
    B, tree = _log_int(rng, 1, 16), rng.random() < 0.7
    L = _log_int(rng, 500, 131072)
    C = 0 if rng.random() < 0.2 else max(8, min(16384, L // rng.randint(20, 64)))
    user = _log_int(rng, 1, min(16384, 1_000_000 // (B * H)))
    keep = min(round(rng.uniform(0.03, 0.3), 3), 1_000_000 / (B * H) / L)
    keys = user + (int(keep * L) if C else 0)
    # rows times keys as in the largest listed case, at most
    T = 1
    want = _log_int(rng, 1, 256 if tree else 2048)
    while T < want and B * H * G * (T + 1) * (keys + (T + 1) // 2) <= 8 * 4 * 2048 * 6000:
        T += 1
    return dict(kind=kind, B=B, H=H, G=G, T=T, tree=tree, L=L, C=C, keep=keep, user=user, page=page, ragged=ragged)


# ---------------------------------------------------------------------------------------------------------------------
# Inputs.
# ---------------------------------------------------------------------------------------------------------------------
def _forest(case, g):
    """Random trees, every draft's parent one of those before it, and how many drafts each sequence has."""
    B, T = case["B"], case["T"]
    u = torch.rand(B, T, generator=g, device="cuda")
    t = torch.arange(T, device="cuda")
    parents = torch.minimum((u * t).long(), (t - 1).clamp(min=0))
    parents[:, 0] = -1
    n = torch.full((B,), T, device="cuda")
    if case["ragged"]:
        n = torch.randint((T + 1) // 2, T + 1, (B,), generator=g, device="cuda")
        n[0] = T
    return parents.int().contiguous(), n.int()


def _pages(case, g, longest, spare, levels=(-7, -5)):
    """A pool with a page table for B sequences of up to `longest` tokens, `spare` pages unused; codes of whole pages, filled or not."""
    P, H, B = case["page"], case["H"], case["B"]
    width = max(1, -(-longest // P))
    used = B * width
    ids = torch.randperm(used + spare, generator=g, device="cuda")[:used].view(B, width).int().contiguous()
    codes = [(64 * torch.randn(used + spare, H, P, D, generator=g, device="cuda")).clamp(-448, 448).to(F8) for _ in range(2)]
    scales = [torch.exp2(torch.randint(*levels, (used + spare, H), generator=g, device="cuda").float()) for _ in range(2)]
    return dict(cK=codes[0], cV=codes[1], cks=scales[0], cvs=scales[1], pages=ids)


def _lengths(case, g, longest):
    n = torch.randint(longest // 2, longest + 1, (case["B"],), generator=g, device="cuda").int()
    n[0] = longest
    return n


def _shares(case):
    """The share of the keys that each (sequence, head) keeps: uneven, and `keep` on average."""
    n = case["B"] * case["H"]
    f = [0.2 + 1.6 * ((r + 1) * 0.6180339887498949 % 1.0) for r in range(n)]
    scale = case["keep"] * n / sum(f)
    return [min(1.0, v * scale) for v in f]


def _kept(case, g):
    """A kept set per (sequence, head): clusters of uneven size, some without keys."""
    H, L, C = case["H"], case["L"], case["C"]
    share = torch.tensor(_shares(case), device="cuda")
    R = share.numel()
    cuts = torch.randint(0, L + 1, (H, C - 1), generator=g, device="cuda").sort(1).values
    ends = torch.cat([cuts, torch.full((H, 1), L, device="cuda")], 1)
    first = torch.cat([torch.zeros(H, 1, dtype=ends.dtype, device="cuda"), cuts], 1)
    size = ends - first
    head = torch.arange(R, device="cuda") % H
    rank = torch.rand(R, C, generator=g, device="cuda").argsort(1).argsort(1)
    keep = (rank < (share * C).round().unsqueeze(1)) & (size[head] > 0)
    order = (~keep).int().sort(dim=1, stable=True).indices
    n = keep.sum(1)
    some = torch.arange(C, device="cuda") < n.unsqueeze(1)
    ranges = torch.stack([torch.where(some, a[head].gather(1, order), 0) for a in (first, size)], 2).int()
    return ranges.contiguous(), n.int(), ranges[:, :, 1].sum(1).int()


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, B = case["kind"], case["B"]
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    if kind == "prepare":
        parents, n = _forest(case, g)
        return dict(parents=parents, n=n, first=torch.randint(0, 100000, (B,), generator=g, device="cuda").int())
    if kind == "accept":
        parents, n = _forest(case, g)
        # few tokens, so that brothers share one at times and several drafts in a row are agreed with
        tokens, target = (torch.randint(0, 3, parents.shape, generator=g, device="cuda").int() for _ in range(2))
        return dict(parents=parents, n=n, tokens=tokens, target=target, seq_len=torch.randint(0, 100000, (B,), generator=g, device="cuda").int())
    H = case["H"]
    if kind == "commit":
        T, path = case["T"], case["path"]
        t = _pages(case, g, case["old"] + (path or T), 3, (-9, -5))
        level = torch.exp(0.5 * randn(2, B, H, 1, 1))                      # heads differ in size
        most = path or T
        n = torch.randint(most // 2, most + 1, (B,), generator=g, device="cuda").int()
        n[0] = most
        t.update(K=(level[0] * randn(B, H, T, D)).half(), V=(level[1] * randn(B, H, T, D)).half(), n=n, path=None,
                 seq_len=torch.randint(0, case["old"] + 1, (B,), generator=g, device="cuda").int())
        if path:
            # ascending drafts, from the first on; behind the accepted ones nothing
            picked = torch.rand(B, T, generator=g, device="cuda").index_fill_(1, torch.zeros(1, dtype=I64, device="cuda"), -1.0).argsort(1)[:, :path].sort(1).values
            t["path"] = torch.full((B, T), -1, dtype=I32, device="cuda")
            t["path"][:, :path] = torch.where(torch.arange(path, device="cuda") < n.unsqueeze(1), picked, -1).int()
        return t
    if kind == "read":
        t = _pages(case, g, case["U"], 3)
        held = _lengths(case, g, case["U"])
        t.update(seq_len=held, first=(held * torch.rand(B, generator=g, device="cuda") * 0.2).int())
        t["first"][0] = 0
        return t
    G, T, L, C = case["G"], case["T"], case["L"], case["C"]
    t = _pages(case, g, case["user"], 2)
    parents, n = _forest(case, g)
    t.update(seq_len=_lengths(case, g, case["user"]), n=n, q=(1.5 * randn(B, H * G, T, D)).half(), K=randn(B, H, T, D).half(),
             V=randn(B, H, T, D).half(), mask=None)
    if case["tree"]:
        t["mask"] = _words(_ancestors(parents.long(), n))
    if not C:
        return t
    ranges, n_ranges, n_keys = _kept(case, g)
    t["most"] = int(n_keys.max())                                          # (for the plain form's buffers)
    t.update(ranges=ranges, n_ranges=n_ranges, n_keys=n_keys,
             K8=(64 * randn(H, L, D)).clamp(-448, 448).to(F8), V8=(64 * randn(H, L, D)).clamp(-448, 448).to(F8),
             ks=torch.exp2(torch.randint(-7, -5, (H, -(-L // BLOCK)), generator=g, device="cuda").float()),
             vs=torch.exp2(torch.randint(-7, -5, (H, -(-L // BLOCK)), generator=g, device="cuda").float()))
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    s = dict(case=case, t=t)
    zeros = lambda *sh, dtype=F16: torch.zeros(*sh, dtype=dtype, device="cuda")  # noqa: E731
    kind, B = case["kind"], case["B"]
    if kind == "prepare":
        T = case["T"]
        s.update(mask=zeros(B, T, -(-T // 32), dtype=I32), positions=zeros(B, T, dtype=I32))
    elif kind == "accept":
        s.update(path=zeros(B, case["T"], dtype=I32), **{k: zeros(B, dtype=I32) for k in ("count", "token", "new_len")})
    elif kind == "read":
        s.update(K=zeros(B, case["H"], case["U"], D), V=zeros(B, case["H"], case["U"], D))
    elif kind == "attend":
        rows = (B, case["H"] * case["G"], case["T"])
        s.update(out=zeros(*rows, D), lse=zeros(*rows, dtype=F32))
    if own:
        _plan(s)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# The framework's calls.
# ---------------------------------------------------------------------------------------------------------------------
def _plan(s):
    """What a program sets up once: the shape, the cache's description, the workspace."""
    from paper_2411_09688_amd import binding as sq
    case, t = s["case"], s["t"]
    kind, B, H, T = case["kind"], case["B"], case.get("H", 1), case.get("T", 1)
    s["sq"] = sq
    if kind in ("commit", "read", "attend"):
        s["cache"] = sq.make_cache(t["cK"], t["cV"], t["cks"], t["cvs"], t["pages"])
    if kind == "attend":
        s["shape"] = sq.make_shape(B, H, case["L"], max(1, case["C"]), case["G"] * T, 0, SM_SCALE)
        s["ws"] = sq.workspace(s["shape"], sq.SQ_CALL_TREE_ATTN_Q8, "cuda:0")
    else:
        s["shape"] = sq.make_shape(B, H, 1, 1, T, case.get("U", 0), SM_SCALE)


def _own(s):
    sq, case, t = s["sq"], s["case"], s["t"]
    kind = case["kind"]
    if kind == "prepare":
        sq.sq_tree_prepare(s["shape"], t["parents"], t["n"], t["first"], s["mask"], s["positions"])
        return dict(mask=s["mask"], positions=s["positions"])
    if kind == "accept":
        sq.sq_tree_accept(s["shape"], t["parents"], t["n"], t["tokens"], t["target"], t["seq_len"], s["count"], s["path"], s["token"], s["new_len"])
        return dict(count=s["count"], path=s["path"], token=s["token"], new_len=s["new_len"])
    if kind == "commit":
        sq.sq_cache_commit(s["shape"], s["cache"], t["seq_len"], t["path"], t["n"], t["K"], t["V"])
        return dict(K8=t["cK"], V8=t["cV"], k_scale=t["cks"], v_scale=t["cvs"])
    if kind == "read":
        sq.sq_cache_read(s["shape"], s["cache"], t["first"], t["seq_len"], s["K"], s["V"])
        return dict(K=s["K"], V=s["V"])
    sq.sq_tree_attn_q8(s["shape"], case["T"], t["q"], t.get("K8"), t.get("V8"), t.get("ks"), t.get("vs"), t.get("ranges"), t.get("n_ranges"),
                       t.get("n_keys"), s["cache"], t["seq_len"], t["K"], t["V"], t["mask"], t["n"] if case["ragged"] else None, s["out"], s["lse"], s["ws"])
    return dict(out=s["out"], lse=s["lse"])


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms.
# ---------------------------------------------------------------------------------------------------------------------
def _ancestors(parents, n):
    """[B, T, T]: whether draft t is draft j or below it, for the first n[b] drafts (the others: nothing)."""
    T = parents.shape[1]
    t = torch.arange(T, device="cuda")
    up = ((parents.unsqueeze(2) == t) | (t.view(-1, 1) == t)).float()
    for _ in range(max(1, (T - 1).bit_length())):                          # (a path of 2^k steps is two of 2^(k - 1))
        up = (torch.bmm(up, up.clone()) > 0).float()
    real = t < n.view(-1, 1)
    return (up > 0) & real.unsqueeze(2) & real.unsqueeze(1)


def _words(bits):
    """[.., T] truth values as 32-bit words [.., ceil(T / 32)]."""
    T = bits.shape[-1]
    w = -(-T // 32)
    b = torch.nn.functional.pad(bits, (0, 32 * w - T)).unflatten(-1, (w, 32)).long()
    v = (b << torch.arange(32, device="cuda")).sum(-1)
    return torch.where(v >= 1 << 31, v - (1 << 32), v).int()


def _rounded(x):
    """To the nearest value of e4m3, ties to even (x within +-448)."""
    step = torch.exp2((torch.frexp(x).exponent - 4).clamp(min=-9).float())
    return torch.round(x / step) * step


def _exponent(amax):
    """The least e with amax <= 448 * 2^e, within the limits."""
    m, e = torch.frexp(amax / 448)
    return torch.where(amax > 0, e - (m == 0.5).int(), E_MIN).clamp(E_MIN, E_MAX)


def _commit_plain(x, t, codes, scales, page, off, real, block, old_end, old):
    """Rounds the rows x [B, n, H, 128] into their pages, with the pages' scales raised where they ask for it.

    page, off [B, n]: where each goes (real: whether it does); block, old_end, old [B]: the page that holds a sequence's last
    tokens so far, how many, and whether it is appended to."""
    pages, H, P, _ = codes.shape
    to, at, ok, y = page.flatten(), off.flatten(), real.flatten(), x.flatten(0, 1)
    amax = torch.zeros(pages, H, device="cuda").index_reduce_(0, to, torch.where(ok.view(-1, 1), y.abs().amax(-1), 0), "amax")
    count = lambda where, what: torch.zeros(pages, 1, dtype=I32, device="cuda").index_add_(0, where, what.int().view(-1, 1))  # noqa: E731
    touched, had = count(to, ok) > 0, count(block, old) > 0
    e_old = torch.frexp(scales).exponent - 1
    e = torch.where(touched, torch.where(had, torch.maximum(e_old, _exponent(amax)), _exponent(amax)), e_old)
    raw = codes.view(U8)
    was = raw[block].view(F8).float()
    again = _rounded(was * torch.exp2((e_old - e)[block].float())[..., None, None])
    mine = (torch.arange(P, device="cuda") < old_end.view(-1, 1)) & old.view(-1, 1)
    raw[block] = torch.where(mine[:, None, :, None], again, was).to(F8).view(U8)
    scales.copy_(torch.exp2(e.float()))
    new = _rounded(y / torch.exp2(e[to].float()).unsqueeze(-1)).to(F8).view(U8)
    raw[to, :, at] = torch.where(ok.view(-1, 1, 1), new, raw[to, :, at])


def _plain(s):
    case, t = s["case"], s["t"]
    kind, B = case["kind"], case["B"]
    if kind in ("prepare", "accept"):
        T = case["T"]
        i = torch.arange(T, device="cuda")
        up = _ancestors(t["parents"].long(), t["n"])
        real = i < t["n"].view(-1, 1)
    if kind == "prepare":
        s["mask"].copy_(_words(up))
        s["positions"].copy_(torch.where(real, t["first"].view(-1, 1) + up.sum(2) - 1, t["first"].view(-1, 1)))
        return dict(mask=s["mask"], positions=s["positions"])
    if kind == "accept":
        parent = t["parents"].long().clamp(min=0)
        right = t["tokens"] == t["target"].gather(1, parent)
        # of brothers with the same token the first one stands for all
        twin = (parent.unsqueeze(2) == parent.unsqueeze(1)) & (t["tokens"].unsqueeze(2) == t["tokens"].unsqueeze(1)) & (i.view(-1, 1) > i) & (i > 0)
        right = ((right & ~twin.any(2)) | (i == 0)) & real
        taken = (~up | right.unsqueeze(1)).all(2) & real                   # a draft and all above it
        count = taken.sum(1).int()
        order = torch.where(taken, i, T).sort(1).values
        s["path"].copy_(torch.where(order < T, order, -1))
        s["count"].copy_(count)
        last = order.gather(1, (count.long() - 1).clamp(min=0).view(-1, 1)).clamp(max=T - 1)
        s["token"].copy_(torch.where(count > 0, t["target"].gather(1, last)[:, 0], -1))
        s["new_len"].copy_(t["seq_len"] + count)
        return dict(count=s["count"], path=s["path"], token=s["token"], new_len=s["new_len"])
    P = case["page"]
    if kind == "commit":
        most = case["path"] or case["T"]
        i = torch.arange(most, device="cuda")
        real = i < t["n"].view(-1, 1)
        slot = torch.where(real, t["seq_len"].view(-1, 1) + i, 0).long()
        # rows that are not written point at a page that nobody has, and change nothing there
        free = torch.ones(t["cK"].shape[0], dtype=I32, device="cuda").index_fill_(0, t["pages"].flatten().long(), 0).argmax()
        page = torch.where(real, t["pages"].long().gather(1, slot // P), free)
        last = (t["seq_len"] // P).clamp(max=t["pages"].shape[1] - 1).long()
        block = t["pages"].gather(1, last.view(-1, 1))[:, 0].long()
        old_end = t["seq_len"] % P
        old = (old_end > 0) & (t["n"] > 0)
        row = i.expand(B, -1) if t["path"] is None else t["path"][:, :most].long().clamp(min=0)
        row = row[:, None, :, None].expand(B, case["H"], most, D)
        for x, codes, scales in ((t["K"], t["cK"], t["cks"]), (t["V"], t["cV"], t["cvs"])):
            _commit_plain(x.gather(2, row).transpose(1, 2).float(), t, codes, scales, page, slot % P, real, block, old_end, old)
        return dict(K8=t["cK"], V8=t["cV"], k_scale=t["cks"], v_scale=t["cvs"])
    if kind == "read":
        U, H = case["U"], case["H"]
        slot = t["first"].view(-1, 1).long() + torch.arange(U, device="cuda")
        real = slot < t["seq_len"].view(-1, 1)
        slot = slot.clamp(max=t["pages"].shape[1] * P - 1)
        at = (t["pages"].long().gather(1, slot // P).unsqueeze(1), torch.arange(H, device="cuda").view(1, -1, 1), (slot % P).unsqueeze(1))
        for out, codes, scales in ((s["K"], t["cK"], t["cks"]), (s["V"], t["cV"], t["cvs"])):
            x = codes.view(U8)[at].view(F8).float() * scales[at[:2]].unsqueeze(-1)
            out.copy_(torch.where(real[:, None, :, None], x, out))
        return dict(K=s["K"], V=s["V"])
    return _attend_plain(s, t, case)


def _attend_plain(s, t, case):
    B, H, G, T, P = (case[k] for k in ("B", "H", "G", "T", "page"))
    R = B * H
    q = t["q"].view(R, G * T, D).float()
    row = torch.arange(R, device="cuda")
    head, seq = row % H, row // H
    # the paged cache
    pos = torch.arange(case["user"], device="cuda")
    page = t["pages"][seq][:, pos // P].long()
    at = (page, head.view(-1, 1), (pos % P).view(1, -1))
    K = [t["cK"].view(U8)[at].view(F8).float() * t["cks"][at[:2]].unsqueeze(-1)]
    V = [t["cV"].view(U8)[at].view(F8).float() * t["cvs"][at[:2]].unsqueeze(-1)]
    ok = [(pos < t["seq_len"][seq].view(-1, 1)).unsqueeze(2)]
    if case["C"]:
        count = t["ranges"][:, :, 1].long()
        ends = count.cumsum(1)
        pos = torch.arange(t["most"], device="cuda").expand(R, -1).contiguous()
        j = torch.searchsorted(ends, pos, right=True).clamp(max=case["C"] - 1)
        key = (t["ranges"][:, :, 0].long().gather(1, j) + pos - (ends - count).gather(1, j)).clamp(0, case["L"] - 1)
        at = (head.view(-1, 1), key)
        K.append(t["K8"].view(U8)[at].view(F8).float() * t["ks"][at[0], key // BLOCK].unsqueeze(-1))
        V.append(t["V8"].view(U8)[at].view(F8).float() * t["vs"][at[0], key // BLOCK].unsqueeze(-1))
        ok.append((pos < t["n_keys"].view(-1, 1)).unsqueeze(2))
    # the drafts
    i = torch.arange(T, device="cuda")
    if case["tree"]:
        sees = (t["mask"].unsqueeze(-1) >> torch.arange(32, device="cuda") & 1).flatten(2)[:, :, :T] > 0       # [B, draft, key]
    else:
        sees = ((i.view(-1, 1) >= i) & (i < t["n"].view(-1, 1, 1)))
    K.append(t["K"].view(R, T, D).float())
    V.append(t["V"].view(R, T, D).float())
    ok.append(sees.transpose(1, 2)[seq].repeat(1, 1, G))                                                      # [R, key, (head, draft)]
    x = [torch.matmul(k, q.transpose(1, 2).contiguous()) * SM_SCALE for k in K]                               # [R, keys, rows]
    x = [torch.where(o, v, -math.inf) for v, o in zip(x, ok)]
    m = torch.stack([v.amax(1) for v in x if v.shape[1]]).amax(0).unsqueeze(1)
    m = torch.where(torch.isfinite(m), m, 0.0)                                                                # (a row without keys)
    p = [torch.exp(v - m) for v in x]
    l = sum(v.sum(1) for v in p)
    o = sum(torch.matmul(v.transpose(1, 2).contiguous(), w) for v, w in zip(p, V))                            # [R, rows, 128]
    real = (i < t["n"].view(-1, 1)).view(B, 1, T)
    out = torch.where(l.unsqueeze(-1) > 0, o / l.unsqueeze(-1), 0.0).view(B, H * G, T, D)
    s["out"].copy_(torch.where(real.unsqueeze(-1), out, s["out"]))
    s["lse"].copy_(torch.where(real, (m[:, 0] + torch.log(l)).view(B, H * G, T), s["lse"]))
    return dict(out=s["out"], lse=s["lse"])


def run(s):
    if own:
        return _own(s)
    return _plain(s)


def work(case):
    """Every input read once, every output written once; of the fixed context the keys that some sequence of a head keeps."""
    kind, B = case["kind"], case["B"]
    T, H = case.get("T", 1), case.get("H", 1)
    some = (0.75 * (B - 1) + 1) / B                        # the mean of lengths between half and all
    if kind == "prepare":
        return dict(bytes=B * T * (4 + 4 + 4.0 * -(-T // 32)) + 8 * B, flops=2.0 * B * T)
    if kind == "accept":
        return dict(bytes=B * T * (3 * 4 + 4.0) + 20 * B, flops=2.0 * B * T)
    if kind == "commit":
        n = B * H * (case["path"] or T) * some
        return dict(bytes=n * 2 * (2 * D + D) + 8 * B, flops=4.0 * n * D)
    if kind == "read":
        n = B * H * case["U"] * some
        return dict(bytes=n * 2 * (2 * D + D) + 8 * B, flops=2.0 * n * D)
    G = case["G"]
    user, drafts = case["user"] * some, T * (some if case["ragged"] else 1.0)
    rows = B * H * G * drafts
    bytes_ = B * H * user * 2 * D + rows * (4 * D + 4) + B * H * drafts * 4 * D
    flops = 4.0 * D * rows * (user + (math.log(T) + 1 if case["tree"] else (T + 1) / 2))
    if case["tree"]:
        bytes_ += B * T * -(-T // 32) * 4
    if case["C"]:
        share = _shares(case)
        kept = [1.0 - math.prod(1.0 - share[b * H + h] for b in range(B)) for h in range(H)]
        bytes_ += sum(kept) * case["L"] * (2 * D + 8 / BLOCK) + sum(share) * case["C"] * 8 + 8 * len(share)
        flops += 4.0 * D * rows * case["L"] * sum(share) / len(share)
    return dict(bytes=bytes_, flops=flops)


# ---------------------------------------------------------------------------------------------------------------------
# The same in 64 bits, from the definitions, one sequence or head after the other.
# ---------------------------------------------------------------------------------------------------------------------
def _powers(lo, hi):
    """2^lo .. 2^hi, made on the host, where they are exact."""
    return torch.tensor([math.ldexp(1.0, e) for e in range(lo, hi + 1)], dtype=F64, device="cuda")


def _nearest(x):
    """The value of e4m3 next to x, looked up among all of them; half way between two, the one of the even place."""
    small = torch.arange(8, dtype=F64, device="cuda") / 512
    grid = torch.cat([small, ((1 + torch.arange(8, dtype=F64, device="cuda") / 8) * _powers(-6, 8).unsqueeze(1)).flatten()])[:127]
    a = x.abs()
    i = torch.searchsorted(grid, a.contiguous(), right=True).sub(1).clamp(0, 125)
    lo, hi = grid[i], grid[i + 1]
    up = (a - lo > hi - a) | ((a - lo == hi - a) & (i % 2 == 1))
    return torch.where(up, hi, lo) * x.sign()


def _scale64(amax):
    """Powers of two tried from small to large: the first that holds amax within 448 times itself."""
    tried = _powers(E_MIN, E_MAX)
    return tried[torch.searchsorted(448 * tried, amax.contiguous()).clamp(max=len(tried) - 1)]


def _line(parents, t):
    """Draft t and those above it."""
    line = [t]
    while 0 <= parents[line[-1]] < line[-1]:
        line.append(parents[line[-1]])
    return line


def exact(case, seed):
    t = _inputs(case, seed)
    kind, B = case["kind"], case["B"]
    if kind == "prepare":
        parents, n, first, T = t["parents"].tolist(), t["n"].tolist(), t["first"].tolist(), case["T"]
        W = -(-T // 32)
        mask, positions = [[[0] * W for _ in range(T)] for _ in range(B)], [[f] * T for f in first]
        for b in range(B):
            for i in range(n[b]):
                line = _line(parents[b], i)
                positions[b][i] = first[b] + len(line) - 1
                for j in line:
                    mask[b][i][j // 32] |= 1 << j % 32
        signed = [[[w - (1 << 32) if w >> 31 else w for w in r] for r in m] for m in mask]
        return dict(mask=torch.tensor(signed, dtype=I32, device="cuda"), positions=torch.tensor(positions, dtype=I32, device="cuda"))
    if kind == "accept":
        parents, n, tokens, target = (t[k].tolist() for k in ("parents", "n", "tokens", "target"))
        found = []
        for b in range(B):
            path = [0][:n[b]]
            while path:
                nxt = [i for i in range(1, n[b]) if parents[b][i] == path[-1] and tokens[b][i] == target[b][path[-1]]]
                if not nxt:
                    break
                path.append(nxt[0])
            found.append(path)
        whole = lambda x: torch.tensor(x, dtype=I32, device="cuda")  # noqa: E731
        count = whole([len(p) for p in found])
        return dict(count=count, path=whole([p + [-1] * (case["T"] - len(p)) for p in found]),
                    token=whole([target[b][p[-1]] if p else -1 for b, p in enumerate(found)]), new_len=t["seq_len"] + count)
    H, P = case["H"], case["page"]
    table = t["pages"].cpu()
    if kind == "commit":
        old, n = t["seq_len"].tolist(), t["n"].tolist()
        found = []
        for x, codes, scales in ((t["K"], t["cK"], t["cks"]), (t["V"], t["cV"], t["cvs"])):
            codes, scales = codes.double(), scales.double()
            for b in range(B):
                rows = x[b].double() if t["path"] is None else x[b].double()[:, t["path"][b, :n[b]].long()]
                done = 0
                while done < n[b]:
                    slot = old[b] + done
                    m, o, page = min(P - slot % P, n[b] - done), slot % P, int(table[b, slot // P])
                    y = rows[:, done:done + m]
                    sc = _scale64(y.abs().amax((1, 2)))
                    if o:
                        sc = torch.maximum(sc, scales[page])
                        codes[page, :, :o] = _nearest(codes[page, :, :o] * (scales[page] / sc).view(H, 1, 1))
                    codes[page, :, o:o + m] = _nearest(y / sc.view(H, 1, 1))
                    scales[page] = sc
                    done += m
            found += [codes, scales]
        return dict(K8=found[0], k_scale=found[1], V8=found[2], v_scale=found[3])
    lengths = t["seq_len"].tolist()

    def held(b, h):
        ids = table[b, :-(-lengths[b] // P)].long().cuda()
        return [(t[a].view(U8)[ids, h].view(F8).double() * t[c][ids, h].double().view(-1, 1, 1)).reshape(-1, D)[:lengths[b]]
                for a, c in (("cK", "cks"), ("cV", "cvs"))]

    if kind == "read":
        out = [torch.zeros(B, H, case["U"], D, dtype=F64, device="cuda") for _ in range(2)]
        first = t["first"].tolist()
        for b in range(B):
            for h in range(H):
                for y, x in zip(out, held(b, h)):
                    y[b, h, :lengths[b] - first[b]] = x[first[b]:]
        return dict(K=out[0], V=out[1])
    G, T = case["G"], case["T"]
    out = torch.zeros(B, H * G, T, D, dtype=F64, device="cuda")
    lse = torch.zeros(B, H * G, T, dtype=F64, device="cuda")
    counts = t["n"].tolist()
    for h in range(H):
        if case["C"]:
            block = torch.arange(case["L"], device="cuda") // BLOCK
            Kf, Vf = (t[a][h].double() * t[c][h].double()[block].unsqueeze(1) for a, c in (("K8", "ks"), ("V8", "vs")))
        for b in range(B):
            n = counts[b]
            k, v = held(b, h)
            if case["C"]:
                first, count = t["ranges"][b * H + h, :, 0].long(), t["ranges"][b * H + h, :, 1].long()
                mark = torch.zeros(case["L"] + 1, dtype=torch.long, device="cuda")
                mark.index_add_(0, first, (count > 0).long()).index_add_(0, first + count, -(count > 0).long())
                kept = mark.cumsum(0)[:-1] > 0
                k, v = torch.cat([Kf[kept], k]), torch.cat([Vf[kept], v])
            if case["tree"]:
                j = torch.arange(n, device="cuda")
                sees = (t["mask"][b, :n].long()[:, j // 32] >> (j % 32) & 1) > 0
            else:
                sees = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
            sees = torch.cat([torch.ones(n, len(k), dtype=torch.bool, device="cuda"), sees], 1)
            k, v = torch.cat([k, t["K"][b, h, :n].double()]), torch.cat([v, t["V"][b, h, :n].double()])
            for i in range(h * G, h * G + G):
                x = (t["q"][b, i, :n].double() @ k.T.contiguous() * SM_SCALE).masked_fill(~sees, -math.inf)
                z = torch.logsumexp(x, 1, keepdim=True)
                out[b, i, :n] = torch.exp(x - z) @ v
                lse[b, i, :n] = z[:, 0]
    return dict(out=out, lse=lse)
