"""From prompts to a verified decode step with two small random models: what a program calls in each layer.

    python examples/prompt_to_step.py

The large model reads its prompts in two chunks (dsbd_kv_append_paged, dsbd_chunk_attention_paged), the small model reads them whole
and then draws drafts: every draft beam is a sequence of its own behind shared prompt pages.  The drafts become a forest,
whose nodes are rotated at their positions (dsbd_forest_positions, dsbd_rotate_qk) and attend in the large model
(dsbd_forest_attention_paged); the verification keeps the output beams and the caches follow them.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2409_16560_b200 as dsbd  # noqa: E402

PAGE, DEV, BF = 64, "cuda", torch.bfloat16


def dev(a, dtype):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=dtype)).to(DEV)


class Model:
    """A decoder of random weights: norm, fused QKV projection, attention, a small MLP."""

    def __init__(self, layers, hidden, Hq, Hkv, d, V, n_pages, seed, max_position=4096):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g, device=DEV) * s[0] ** -0.5).to(BF)
        self.layers, self.Hq, self.Hkv, self.d, self.scale = layers, Hq, Hkv, d, d ** -0.5
        self.embed = torch.randn(V, hidden, generator=g, device=DEV).to(BF)
        self.qkv = [w(hidden, (Hq + 2 * Hkv) * d) for _ in range(layers)]
        self.out = [w(Hq * d, hidden) for _ in range(layers)]
        self.up, self.down = ([w(*s) for _ in range(layers)] for s in ((hidden, 2 * hidden), (2 * hidden, hidden)))
        self.unembed = w(hidden, V) * 3
        table = dsbd.rope_table(max_position, d, base=10000.0)
        norm = lambda: 1 + 0.1 * torch.randn(d, generator=g, device=DEV)
        self.rope = [dsbd.Rope(table, layout="half", q_norm=norm(), k_norm=norm()) for _ in range(layers)]
        # a page id means the same slot in the pools of every layer; zeros, so that all rows are finite
        self.k_pool = torch.zeros(layers, n_pages, Hkv, PAGE, d, dtype=BF, device=DEV)
        self.v_pool = torch.zeros_like(self.k_pool)
        self.free = list(range(n_pages))

    def pages(self, n):
        taken, self.free = self.free[:n], self.free[n:]
        return taken

    def _project(self, x, l):
        y = x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)
        q, k, v = (y.to(BF) @ self.qkv[l]).split([self.Hq * self.d, self.Hkv * self.d, self.Hkv * self.d], 1)
        return q.unflatten(1, (self.Hq, self.d)), k.unflatten(1, (self.Hkv, self.d)), v.unflatten(1, (self.Hkv, self.d))

    def _finish(self, x, att, l):
        x = x + att.flatten(1) @ self.out[l]
        return x + torch.relu(x @ self.up[l]) @ self.down[l]

    def read(self, tokens, chunk, status):
        """New tokens of some sequences through all layers, behind what is cached; logits of every new token."""
        x = self.embed[tokens]
        for l in range(self.layers):
            q, k, v = self._project(x, l)
            q, _ = dsbd.kv_append_paged(chunk, k, v, self.k_pool[l], self.v_pool[l], rope=self.rope[l], q=q, status=status)
            att, _ = dsbd.chunk_attention_paged(chunk, self.Hq, self.Hkv, self.d, self.scale, q, self.k_pool[l], self.v_pool[l],
                                                status=status)
            x = self._finish(x, att, l)
        return (x @ self.unembed).float()

    def read_forest(self, forest, tokens, tables, status):
        """The nodes of a forest through all layers; logits of every node and the nodes' keys and values."""
        table, page_off, prefix_off, prefix_off_host = tables
        position, _ = dsbd.forest_positions(forest, prefix_off, status=status)
        x, ks, vs = self.embed[tokens], [], []
        for l in range(self.layers):
            q, k, v = self._project(x, l)
            q, k, _ = dsbd.rotate_qk(q, k, position, self.rope[l], status=status)
            v = v.contiguous()
            att, _ = dsbd.forest_attention_paged(forest, self.Hq, self.Hkv, self.d, self.scale, q, k, v, self.k_pool[l],
                                                 self.v_pool[l], table, page_off, prefix_off, prefix_off_host, status=status)
            x = self._finish(x, att, l)
            ks.append(k)
            vs.append(v)
        return (x @ self.unembed).float(), torch.stack(ks), torch.stack(vs)


def chunk(new, old, tables):
    """A Chunk of new[b] tokens behind old[b] cached ones, pages tables[b]."""
    off = lambda n: np.concatenate([[0], np.cumsum(n)])
    no, po, to = off(new), off(old), off([len(t) for t in tables])
    return dsbd.Chunk(dev(no, np.int32), no, dev(po, np.int64), po, dev(np.concatenate(tables), np.int32), dev(to, np.int64))


def run(lengths=(150, 65), gamma=3, W_S=4, V=1000, seed=0):
    """One decode step of len(lengths) requests, one input beam each.  Returns what a test wants to look at."""
    rng = np.random.default_rng(seed)
    R = len(lengths)
    prompts = [rng.integers(0, V, n) for n in lengths]
    large = Model(2, 256, 8, 2, 128, V, 64, seed)
    small = Model(1, 128, 4, 4, 64, V, 128, seed + 1)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    need = lambda n: -(-n // PAGE)
    # a prompt's last token is the root of the request's draft tree: everything before it goes to the caches
    cached = [n - 1 for n in lengths]
    tables = [large.pages(need(n)) for n in cached]
    first = [n // 2 for n in cached]
    for new, old in ((first, [0] * R), ([n - f for n, f in zip(cached, first)], first)):
        tok = np.concatenate([p[o:o + n] for p, o, n in zip(prompts, old, new)])
        large.read(dev(tok, np.int64), chunk(new, old, tables), status)
    small_tables = [small.pages(need(n)) for n in cached]
    small.read(dev(np.concatenate([p[:-1] for p in prompts]), np.int64), chunk(cached, [0] * R, small_tables), status)

    # ---- the small model draws gamma layers of W_S drafts a request; a beam is the request's root token and the draws on its path
    def small_logits(paths, request):
        """Next-token logits behind every path: each is a sequence with pages of its own from the prompt's last one on."""
        own = []
        for r, path in zip(request, paths):
            whole = cached[r] // PAGE
            t = small_tables[r][:whole] + small.pages(need(cached[r] + len(path)) - whole)
            if cached[r] % PAGE:
                for pool in (small.k_pool, small.v_pool):
                    pool[:, t[whole]] = pool[:, small_tables[r][whole]]
            own.append(t)
        c = chunk([len(p) for p in paths], [cached[r] for r in request], own)
        logits = small.read(dev(np.concatenate(paths), np.int64), c, status)
        small.free = small.free + [p for r, t in zip(request, own) for p in t[cached[r] // PAGE:]]
        return logits[dev(np.cumsum([len(p) for p in paths]) - 1, np.int64)].contiguous()

    rbo = np.arange(R + 1)
    prm = dict(V=V, temperature=1.0, seed=7, step=0)
    paths, request = [np.array([p[-1]]) for p in prompts], list(range(R))
    off, score = rbo, torch.zeros(R, device=DEV)
    zq, draws = [small_logits(paths, request)], []
    for l in range(1, gamma + 1):
        out_off = W_S * np.arange(R + 1)
        d = dsbd.draft_layer(dev(off, np.int32), off, prm, l, W_S, zq[-1], score, dev(out_off, np.int32), R * W_S, status=status)
        parent, token = d["out_parent"].cpu().numpy(), d["out_token"].cpu().numpy()
        paths = [np.append(paths[p], t) for p, t in zip(parent, token)]
        request = [request[p] for p in parent]
        off, score = out_off, d["out_logq"]
        draws.append((d["out_parent"], d["out_token"]))
        zq.append(small_logits(paths, request))

    # ---- the forest through the large model
    forest, node_of_draw, _ = dsbd.forest_build(dev(rbo, np.int32), rbo, gamma, W_S, torch.stack([p for p, _ in draws]),
                                                torch.stack([t for _, t in draws]), status=status, exact=True)
    roots = forest.dev["beam_node_off"][:-1].long()
    tokens = forest.dev["token"].clone()
    tokens[roots] = dev([p[-1] for p in prompts], np.int32)
    poff = np.concatenate([[0], np.cumsum(cached)])
    table, page_off = dev(np.concatenate(tables), np.int32), dev(np.concatenate([[0], np.cumsum([len(t) for t in tables])]), np.int64)
    prefix_off = dev(poff, np.int64)
    zp, k_new, v_new = large.read_forest(forest, tokens.long(), (table, page_off, prefix_off, poff), status)
    zq_nodes = torch.empty(forest.N, V, device=DEV)
    zq_nodes[roots] = zq[0]
    for l in range(gamma):
        zq_nodes[node_of_draw[l].long()] = zq[l + 1]

    # ---- verification, and the caches of the output beams
    arrays = dict(R=R, beam_node_off=forest.dev["beam_node_off"].cpu().numpy(), req_beam_off=rbo)
    vprm = dict(prm, thresh=0.6, W_min=1, W_max=3, W_nom=3)
    out_off = dsbd.default_out_off(arrays, vprm)
    out = dsbd.alloc_verify_out(forest, out_off, DEV)
    dsbd.verify_step(forest, vprm, zp, zq_nodes, torch.zeros(R, device=DEV), torch.zeros(R, device=DEV), out, status=status)
    free = np.zeros(64, np.int32)
    free[:len(large.free)] = large.free
    res = dsbd.kv_commit_paged(forest, large.Hkv, large.d, out["out_off"], out["out_width"], out["out_parent"], out["out_root_beam"],
                               out["out_logp"], k_new, v_new, large.k_pool, large.v_pool, table, page_off, prefix_off, poff,
                               dev(free, np.int32), dev([len(large.free)], np.int32), n_slots=int(out_off[-1]), table_capacity=64,
                               status=status)
    torch.cuda.synchronize()
    return dict(large=large, prompts=prompts, forest=forest, tokens=tokens, zp=zp, out=out, commit=res, status=int(status.item()),
                need=need, out_off=out_off)


def main():
    r = run()
    out, off = r["out"], r["out_off"]
    for i in range(len(r["prompts"])):
        w = int(out["out_width"][i])
        s = slice(int(off[i]), int(off[i]) + w)
        print("request %d: %d prompt tokens, stopped in layer %d, %d beams, tokens %s, cache lengths %s" % (
            i, len(r["prompts"][i]), int(out["l_last"][i]), w, out["out_token"][s].tolist(),
            [int(x) for x in (r["commit"]["new_prefix_off"][1:] - r["commit"]["new_prefix_off"][:-1])[int(r["commit"]["new_req_beam_off"][i]):
                                                                 int(r["commit"]["new_req_beam_off"][i + 1])]]))
    print("status", r["status"])


if __name__ == "__main__":
    main()
