"""Trees of drafted tokens, pools of counted pages and the normalised rotation as the header defines them, in plain loops on the CPU; shares no
code with the kernels."""
import torch

import q8_reference as R


def chains(parent):
    """For every node of one tree itself and the nodes above it, in order; a parent that is not before its node counts as none."""
    out = []
    for t, p in enumerate(int(x) for x in parent):
        out.append((out[p] if 0 <= p < t else []) + [t])
    return out


def random_tree(g, B, L, kind="mixed"):
    """int32 [B, L]"""
    parent = torch.full((B, L), -1, dtype=torch.int32)
    for b in range(B):
        for t in range(1, L):
            if kind == "chain":
                parent[b, t] = t - 1
            elif kind == "roots":
                parent[b, t] = -1 - t
            elif kind == "star":
                parent[b, t] = 0
            else:
                parent[b, t] = t - 1 if torch.rand(1, generator=g) < 0.4 else int(torch.randint(-1, t, (1,), generator=g))
    return parent


def attend(cache, q, k, v, flags, parent, scale):
    """q [B, Hq, L, D], k, v [B, Hkv, L, D] (turned), flags [B, Hkv, L] bool, parent [B, L] -> float64 [B, Hq, L, D]"""
    B, Hq, L, D = q.shape
    G = Hq // cache.Hkv
    out = torch.empty(B, Hq, L, D, dtype=torch.float64)
    for u in range(B * cache.Hkv):
        b, h = divmod(u, cache.Hkv)
        K, V, own_k, own_v = cache.rows(u, 0), cache.rows(u, 1), k[b, h].double(), v[b, h].double()
        for t, chain in enumerate(chains(parent[b])):
            mine = [x for x in chain[:-1] if flags[b, h, x]] + [t]
            kk, vv = torch.cat([K, own_k[mine]]), torch.cat([V, own_v[mine]])
            s = q[b, h * G:(h + 1) * G, t].double() @ kk.T * scale
            out[b, h * G:(h + 1) * G, t] = torch.softmax(s, dim=1) @ vv if kk.shape[0] > 1 else vv.expand(G, D)
    return out


def path(parent, last):
    """The accepted node and those above it, in order."""
    return chains(parent)[int(last)] if 0 <= int(last) < parent.shape[0] else []


# ---- pools ----
def count(tables, n_pages):
    """How many entries of the tables name each page."""
    ref = torch.zeros(n_pages, dtype=torch.int32)
    for page in tables:
        for p in page.reshape(-1).tolist():
            if 0 <= p < n_pages:
                ref[p] += 1
    return ref


def reserve(page, length, ref, rows):
    """page, ref written; whether all found room"""
    n, all_there = ref.numel(), True
    U, blocks = page.shape
    free = iter([p for p in range(n) if ref[p] == 0])
    for u in range(U):
        end = (int(length[u]) + rows) // R.BLOCK
        all_there &= end <= blocks
        for j in range(int(length[u]) // R.BLOCK, min(end, blocks)):
            if not 0 <= int(page[u, j]) < n:
                p = next(free, None)
                if p is None:
                    all_there = False
                else:
                    page[u, j] = p
                    ref[p] = 1
    return all_there


def fork(src, parent, dst_page, dst_len, ref, H):
    """src = (page, len); dst_page, dst_len, ref written; the unit of src (None: empty) whose tails each unit of dst has"""
    n, tails = ref.numel(), []
    for u in range(dst_page.shape[0]):
        b, h = divmod(u, H)
        for p in dst_page[u].tolist():
            if 0 <= p < n:
                ref[p] -= 1
        dst_page[u] = -1
        some = 0 <= int(parent[b]) < src[0].shape[0] // H
        v = int(parent[b]) * H + h if some else None
        tails.append(v)
        dst_len[u] = src[1][v] if some else 0
        for j in range(int(dst_len[u]) // R.BLOCK):
            p = int(src[0][v, j])
            if 0 <= p < n:
                dst_page[u, j] = p
                ref[p] += 1
    return tails


def compact(ref):
    """(new numbers, counts, pages in use)"""
    used = [p for p in range(ref.numel()) if ref[p] != 0]
    n = len(used)
    moved = torch.full_like(ref, -1)
    holes = [p for p in range(n) if ref[p] == 0]
    for p in used:
        moved[p] = p if p < n else holes.pop(0)
    new = torch.zeros_like(ref)
    for p in used:
        new[moved[p]] = ref[p]
    return moved, new, n


# ---- normalised rotation ----
def normed64(x, w, eps):
    x = x.double()
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
