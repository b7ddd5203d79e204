"""Device-buffer plumbing around the C ABI for the tests and the benchmark: uploads the seeded
synthetic model, allocates the KV buffer, workspace and outputs as torch tensors, and calls the
library.  No arithmetic of the method happens here."""
from __future__ import annotations

import torch

from . import binding as vb


class Rollout:
    """One model on one GPU plus the buffers for a (B, S, A) rollout problem."""

    def __init__(self, synth_model, max_batch: int, max_seq: int, device="cuda:0", with_value=True,
                 value_b: float = 0.0, value_dim: int = 1, prepack: bool = True):
        self.shape = synth_model.shape
        self.device = torch.device(device)
        assert str(synth_model.device).startswith("cuda"), "weights must be generated on the GPU"
        self.value_dim = value_dim
        self.cfg = vb.make_config(self.shape, max_batch, max_seq, value_dim)
        layers = [synth_model.layer(l) for l in range(self.shape.n_layers)]
        self.embed = synth_model.embed()
        self.model = vb.DeviceModel(self.cfg, self.embed, synth_model.lm_head(), synth_model.final_norm(),
                                    layers, synth_model.value_w(value_dim) if with_value else None, value_b,
                                    synth_model.value_bias(value_dim) if with_value and value_dim > 1 else None)
        self._bufs = {}
        # repacked projection weights for the multi-row forwards (bf16 models with tile-aligned widths)
        self.packed = None
        nbytes = vb.vla_prepack_bytes(self.cfg)
        if nbytes and prepack:
            self.packed = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            vb.vla_prepack(self.model.handle, self.packed)
            torch.cuda.synchronize(self.device)

    def _buf(self, name, nbytes):
        t = self._bufs.get(name)
        if t is None or t.numel() < nbytes:
            self._bufs[name] = t = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        return t

    def _value_out(self, n):
        shape = (n,) if self.value_dim == 1 else (n, self.value_dim)
        return torch.empty(*shape, dtype=torch.float32, device=self.device)

    def kv(self, B, max_pos, lane=0):
        return self._buf(f"kv{lane}", vb.vla_kv_bytes(self.cfg, B, max_pos))

    # `lane` selects a private KV buffer and workspace, so that calls on different streams can overlap.
    def prefill(self, patch, ids, want_value=True, stream=None, lane=0):
        B, P = patch.shape[0], patch.shape[1]
        T = ids.shape[1]
        kv = self.kv(B, self.cfg.max_seq, lane)
        ws = self._buf(f"ws{lane}", vb.vla_workspace_bytes(self.cfg, vb.VLA_ENTRY_PREFILL, B, P + T, 0))
        h_last = torch.empty(B, self.shape.hidden, dtype=torch.float32, device=self.device)
        value = self._value_out(B) if want_value else None
        vb.vla_prefill(self.model.handle, kv, ws, patch, ids, B, P, T, h_last, value, stream)
        return h_last, value

    def decode(self, h_last, S, A, mode=0, slot_embed=None, temperature=1.0, gumbel=None,
               want_logits=True, stream=None, lane=0):
        B = h_last.shape[0]
        kv = self.kv(B, self.cfg.max_seq, lane)
        ws = self._buf(f"ws{lane}", vb.vla_workspace_bytes(self.cfg, vb.VLA_ENTRY_DECODE, B, S, A))
        dev = self.device
        bins = torch.empty(B, A, dtype=torch.int32, device=dev)
        logp = torch.empty(B, A, dtype=torch.float32, device=dev)
        ent = torch.empty(B, A, dtype=torch.float32, device=dev)
        logits = torch.empty(B, A, 256, dtype=torch.float32, device=dev) if want_logits else None
        vb.vla_decode_actions(self.model.handle, kv, ws, h_last, B, S, A, mode, slot_embed, temperature,
                              gumbel, bins, logp, ent, logits, stream)
        return bins, logp, ent, logits

    def recompute(self, patch, ids, bins, A, mode=0, slot_embed=None, temperature=1.0, want_value=True,
                  want_logits=True, stream=None):
        N, P = patch.shape[0], patch.shape[1]
        T = ids.shape[1]
        ws = self._buf("ws0", vb.vla_workspace_bytes(self.cfg, vb.VLA_ENTRY_RECOMPUTE, N, P + T, A))
        dev = self.device
        logp = torch.empty(N, A, dtype=torch.float32, device=dev)
        ent = torch.empty(N, A, dtype=torch.float32, device=dev)
        value = self._value_out(N) if want_value else None
        logits = torch.empty(N, A, 256, dtype=torch.float32, device=dev) if want_logits else None
        vb.vla_logprob_recompute(self.model.handle, ws, patch, ids, bins, N, P, T, A, mode, slot_embed,
                                 temperature, logp, ent, value, logits, stream)
        return logp, ent, value, logits


    def backward(self, patch, ids, bins, coef, A, lora, rank, scale, mode=0, slot_embed=None, temperature=1.0, stream=None,
                 keep_activations=False):
        """LoRA gradients of sum(coef * logp): lora[l][p] = (a, b) device tensors in the storage dtype.  Returns
        (grads, logp) with grads[l][p] = (da, db) fp32 device tensors.  keep_activations: hand the library the larger
        workspace with which it keeps every layer's activations instead of running all but the top ones a second time."""
        N, P = patch.shape[0], patch.shape[1]
        T = ids.shape[1]
        size = vb.vla_backward_keep_workspace_bytes if keep_activations else vb.vla_backward_workspace_bytes
        ws = self._buf("ws_bw", size(self.cfg, N, P + T, A, rank))
        grads = [{p: (torch.empty(f[0].shape, dtype=torch.float32, device=self.device),
                      torch.empty(f[1].shape, dtype=torch.float32, device=self.device)) for p, f in layer.items()}
                 for layer in lora]
        logp = torch.empty(N, A, dtype=torch.float32, device=self.device)
        vb.vla_logprob_backward(self.model.handle, ws, patch, ids, bins, coef, N, P, T, A, mode, slot_embed, temperature,
                                rank, scale, keep_activations, lora, grads, logp, stream)
        return grads, logp


class PagedRollout:
    """Rollouts of environments whose prefixes have any lengths, on a paged cache of ``n_pages`` pages a layer: one ragged prefill, then
    action tokens sampled with top-k, top-p and min-p.  Pages are taken from the free ones as sequences grow; a prefill frees all.  A call that is refused
    changes nothing: the sequences that are there go on.  Work goes to
    ``stream``, or to the current one; one that is not the last call's, or the one the arguments were made on, has to wait for it first.
    Several on one ``run`` share its weights alone: their calls may overlap on different streams.

    ``weigh``: the weight that rows give each position is summed, for ``evict`` (forwards are then of all sequences, and give no h_last or value).  ``decode`` reads
    ``select`` pages a row and head where that is given; ``decode_drafts`` takes trees of drafted tokens through one forward."""

    def _used(self, t):
        """t, which is not given out again on the stream it was made on before the current one is through with it."""
        if t.is_cuda:
            t.record_stream(torch.cuda.current_stream(self.device))
        return t

    def _buf(self, name, nbytes):
        return self._used(Rollout._buf(self, name, nbytes))

    def __init__(self, run: Rollout, n_pages: int, page_size: int = 16, weigh: bool = False):
        s = run.shape
        self.run, self.page_size = run, page_size
        self.device, self._bufs = run.device, {}
        self.pools = [torch.zeros(s.n_layers, n_pages, s.n_heads, page_size, s.head_dim, dtype=s.torch_dtype, device=run.device) for _ in range(2)]
        self.cache = vb.make_paged_cache(self.pools[0][0], self.pools[1][0])
        self.layer_stride = self.pools[0][0].numel()
        self.n_pages = n_pages
        self.shared_len = 0
        self.weigh, self.mass, self.shift = weigh, None, []          # shift: how many positions a sequence has lost
        self._hold(self._fresh(0))

    def _fresh(self, n_seq):
        """Of n_seq sequences without a position: their pages, their lengths, the free pages."""
        return [[] for _ in range(n_seq)], [0] * n_seq, list(range(self.n_pages - 1, -1, -1))

    def _hold(self, held):
        self.pages, self.length, self.free = held

    def _grown(self, held, seqs, rows):
        """`held` with rows[i] more positions for seqs[i]; what is given stays as it is."""
        pages, length, free = held
        wanted = [max(0, -(-(length[s] + n) // self.page_size) - len(pages[s])) for s, n in zip(seqs, rows)]
        if sum(wanted) > len(free):
            raise ValueError(f"{sum(wanted)} pages wanted, {len(free)} of {self.n_pages} free")
        length, left = list(length), len(free) - sum(wanted)
        for s, n in zip(seqs, rows):
            length[s] += n
        if left < len(free):
            pages, more, free = list(pages), iter(free[left:][::-1]), free[:left]
            for s, n in zip(seqs, wanted):
                pages[s] = pages[s] + [next(more) for _ in range(n)]
        return pages, length, free

    def _int(self, values):
        return torch.tensor(values, dtype=torch.int32, device=self.run.device)

    def forward(self, seqs, ids, rows, patch=None, prefix_len=None, shared_len=0, want_value=False, stream=None):
        """New rows for the sequences ``seqs``: rows[i] of them for seqs[i], ids of all together.  Returns (h_last, logits, value)."""
        with torch.cuda.stream(stream):
            return self._forward(seqs, ids, rows, patch, prefix_len, shared_len, want_value)

    def _batch(self, held, seqs, rows):
        """The batch of new rows for seqs as `held` has them."""
        pages, length, _ = held
        entries = max(1, max(len(pages[s]) for s in seqs))
        table = self._int([pages[s] + [-1] * (entries - len(pages[s])) for s in seqs])
        starts = [0]
        for n in rows:
            starts.append(starts[-1] + n)
        return vb.make_paged_batch(self._int(starts), self._int([length[s] for s in seqs]), table, starts[-1], max(rows), max(length[s] for s in seqs))

    def _plan(self, held, seqs, rows, shared_len):
        """... and the workspace it takes: all that can be refused of it for its sizes."""
        batch = self._batch(held, seqs, rows)
        return batch, vb.vla_forward_paged_workspace_bytes(self.run.cfg, self.cache, batch, shared_len)

    def _room(self, n, most):
        """The summed weights of n sequences, with room for `most` positions, for the current stream."""
        s, have = self.run.shape, 0 if self.mass is None or self.mass.shape[1] != n else self.mass.shape[3]
        if have:
            self._used(self.mass)
        if have < most:                                      # (a thousand more at a time)
            more = torch.zeros(s.n_layers, n, s.n_heads, -(-most // 1024) * 1024, device=self.device)
            if have:
                more[:, :, :, :have] = self.mass
            self.mass = more
        return self.mass

    def _run_rows(self, held, seqs, rows, ids, patch=None, shared_len=0, depth=None, **options):
        """Logits of every new row, by vla_forward_paged_rows.  depth [n_rows]: of the rows' positions behind their sequences, where these are not one behind the other."""
        s, n_all = self.run.shape, len(held[0])
        batch = self._batch(held, seqs, rows)
        if depth is not None or any(self.shift):
            shift = [self.shift[q] if q < len(self.shift) else 0 for q in seqs]
            first = torch.repeat_interleave(self._int([held[1][q] - n + z for q, n, z in zip(seqs, rows, shift)]), self._int(rows), output_size=batch.n_rows)
            if depth is None:
                depth = torch.cat([torch.arange(n, dtype=torch.int32, device=self.device) for n in rows])
            options["position"] = (first + depth).to(torch.int32)
        if self.weigh and options.get("seen") is None:
            if list(seqs) != list(range(n_all)):
                raise ValueError(f"sequences {list(seqs)}: weights are summed for all {n_all} at once")
            options["mass"] = self._room(n_all, batch.max_len)
        plan = vb.make_paged_rows(**options)
        size = vb.vla_forward_paged_rows_workspace_bytes(self.run.cfg, self.cache, batch, plan, shared_len)
        logits = torch.empty(batch.n_rows, vb.VLA_N_BINS, dtype=torch.float32, device=self.device)
        vb.vla_forward_paged_rows(self.run.model.handle, self.cache, self.layer_stride, s.n_layers, batch, plan, ids, self._buf("ws_rows", size), logits, patch, shared_len)
        return logits

    def _run(self, plan, ids, patch, prefix_len, shared_len, want_value):
        run, dev = self.run, self.run.device
        batch, ws_bytes = plan
        h = torch.empty(batch.n_seq, run.shape.hidden, dtype=torch.float32, device=dev)
        logits = torch.empty(batch.n_seq, vb.VLA_N_BINS, dtype=torch.float32, device=dev)
        value = run._value_out(batch.n_seq) if want_value else None
        vb.vla_forward_paged(run.model.handle, self.cache, self.layer_stride, batch, ids, self._buf("ws_paged", ws_bytes), h, patch, prefix_len, shared_len, logits, value)
        return h, logits, value

    def _forward(self, seqs, ids, rows, patch=None, prefix_len=None, shared_len=0, want_value=False, held=None, select=0, bounds=None):
        held = held or (self.pages, self.length, self.free)
        if not len(seqs) or len(set(seqs)) != len(seqs) or min(seqs) < 0 or max(seqs) >= len(held[0]):
            raise ValueError(f"sequences {list(seqs)}: wanted some of the {len(held[0])}, each once")
        if len(rows) != len(seqs) or min(rows) < 0 or sum(rows) != ids.numel():
            raise ValueError(f"{ids.numel()} ids in rows {list(rows)} for {len(seqs)} sequences")
        held = self._grown(held, seqs, rows)
        if self.weigh or select or any(self.shift[s] for s in seqs if s < len(self.shift)):
            more = dict(bounds=bounds, n_select=select, first=int(select > 2), recent=min(2, select)) if select else {}
            logits = self._run_rows(held, seqs, rows, ids, patch, 0 if select else shared_len, prefix_len=prefix_len, **more)
            last, n = [], 0
            for r in rows:
                n += r
                last.append(n - 1)
            out = None, torch.where(self._int(rows)[:, None] > 0, logits[self._int(last).long().clamp(min=0)], 0.0), None          # (no row: as of a row of zeros)
        else:
            out = self._run(self._plan(held, seqs, rows, shared_len), ids, patch, prefix_len, shared_len, want_value)
        self._hold(held)                                     # (nothing has changed where any of this was refused)
        return out

    def prefill(self, patches, ids, see_patches=False, stream=None):
        """patches[i] [P_i, hidden] (or None) and ids[i] [T_i] of environment i.  see_patches: an environment's patches see each other
        both ways, its instruction sees what is before it.  Returns (h_last, logits, value)."""
        with torch.cuda.stream(stream):
            return self._prefill(patches, ids, see_patches)

    def _prefill(self, patches, ids, see_patches=False):
        dev = self.run.device
        if not len(ids) or len(patches) != len(ids):
            raise ValueError(f"patches of {len(patches)} and ids of {len(ids)} sequences")
        n_patch = [0 if p is None else p.shape[0] for p in patches]
        parts, seen = [], 0
        for n, t in zip(n_patch, ids):
            parts += [-1 - torch.arange(seen, seen + n, dtype=torch.int32, device=dev), t.to(torch.int32)]
            seen += n
        patch = [p for p in patches if p is not None and p.shape[0]]
        before, self.shift, self.mass = (self.shift, self.mass), [], None          # (a prefill's positions are their places)
        try:
            out = self._filled(n_patch, ids, parts, patch, see_patches)
        except Exception:
            self.shift, self.mass = before
            raise
        self.shared_len, self.shift = 0, [0] * len(ids)
        return out

    def _filled(self, n_patch, ids, parts, patch, see_patches):
        return self._forward(list(range(len(ids))), torch.cat(parts), [n + t.numel() for n, t in zip(n_patch, ids)], torch.cat(patch) if patch else None,
                             self._int(n_patch) if see_patches else None, 0, self.run.model._keep[4] is not None, self._fresh(len(ids)))

    def prefill_group(self, patch, ids, group: int, stream=None):
        """One observation (patch or None, ids) for ``group`` rollouts: its whole pages are computed and kept once, what is behind them once per rollout."""
        with torch.cuda.stream(stream):
            return self._prefill_group(patch, ids, group)

    def _prefill_group(self, patch, ids, group):
        if group < 1:
            raise ValueError(f"a group of {group} rollouts")
        if self.weigh:
            raise ValueError("a group shares pages, which no rollout of it may cut: weights are not summed for one")
        patch = None if patch is None else patch.contiguous()
        n_patch = 0 if patch is None else patch.shape[0]
        n = n_patch + ids.numel()
        shared = (n - 1) // self.page_size * self.page_size
        rows, others = [n - shared] * (group - 1), list(range(1, group))
        first = self._grown(self._fresh(1), [0], [n])
        held = first
        if others:                                           # both halves are laid out before either runs
            pages, length, free = first
            held = self._grown((pages + [pages[0][:shared // self.page_size] for _ in others], length + [shared] * len(others), free), others, rows)
            rest = self._plan(held, others, rows, shared)
            self._buf("ws_paged", rest[1])
        value = self.run.model._keep[4] is not None
        every = torch.cat([-1 - torch.arange(n_patch, dtype=torch.int32, device=self.run.device), ids.to(torch.int32)])
        out = self._run(self._plan(first, [0], [n], 0), every, patch, None, 0, value)
        if others:
            more = self._run(rest, every[shared:].repeat(group - 1), patch, None, shared, value)
            out = tuple(None if a is None else torch.cat([a, b]) for a, b in zip(out, more))
        self._hold(held)
        self.shared_len, self.shift, self.mass = shared if others else 0, [0] * group, None
        return out

    def decode(self, logits, n_tokens: int, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=None, stream=None, select=0):
        """n_tokens action tokens of every sequence from the first one's logits; u [n_tokens, n_seq] in [0, 1), or None: the largest.
        select: pages that a row and head reads, the first, the last two and those with the largest bounds of its scores (0: all).
        Returns bins, logp (under softmax(z / temperature)), logp_kept (among the kept bins), logits, each [n_seq, n_tokens, ...]."""
        with torch.cuda.stream(stream):
            return self._decode(logits, n_tokens, temperature, top_k, top_p, min_p, u, select)

    def _all_bounds(self):
        """Bounds of all pages that are held."""
        s, every = self.run.shape, list(range(len(self.pages)))
        bounds = torch.zeros(s.n_layers, self.n_pages, s.n_heads, 2, s.head_dim, dtype=s.torch_dtype, device=self.device)
        batch = self._batch((self.pages, self.length, self.free), every, self.length)
        for l in range(s.n_layers):
            vb.vla_paged_bounds(vb.make_paged_cache(self.pools[0][l], self.pools[1][l]), batch, bounds[l])
        return bounds

    def evict(self, keep: int, first=0, recent=0, stream=None):
        """Cuts every layer and head of every sequence that holds more to ``keep`` positions: the first ``first``, the last ``recent`` and those that rows gave most weight.  Later rows are
        rotated by the positions they would have had.  Takes free pages for what stays before it gives the old ones back."""
        with torch.cuda.stream(stream):
            self._evict(keep, first, recent)

    def _evict(self, keep, first, recent):
        if not self.weigh or self.mass is None:
            raise ValueError("no weights were summed (weigh)")
        if keep < 1 or first < 0 or recent < 0 or first + recent > keep:
            raise ValueError(f"keep {keep}, first {first}, recent {recent}")
        s, n, each = self.run.shape, len(self.pages), -(-keep // self.page_size)
        cut = [l > keep for l in self.length]
        if sum(cut) * each > len(self.free):
            raise ValueError(f"{sum(cut) * each} pages wanted, {len(self.free)} of {self.n_pages} free")
        free = list(self.free)
        pages = [[free.pop() for _ in range(each)] if c else p for c, p in zip(cut, self.pages)]
        to_table = self._int([(p + [-1] * each)[:each] for p in pages])
        batch = self._batch((self.pages, self.length, self.free), list(range(n)), [0] * n)
        kept, mass = torch.empty(n, s.n_heads, keep, dtype=torch.int32, device=self.device), self._room(n, max(self.length))
        for l in range(s.n_layers):
            cache = vb.make_paged_cache(self.pools[0][l], self.pools[1][l])
            vb.vla_paged_evict(cache, batch, mass[l], first, recent, to_table, kept, mass[l])
        self.shift = [z + max(0, l - keep) for z, l in zip(self.shift, self.length)]
        used = {q for p in pages for q in p}
        self._hold((pages, [min(l, keep) for l in self.length], [q for q in range(self.n_pages - 1, -1, -1) if q not in used]))

    def decode_drafts(self, tokens, parents, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=None, stream=None):
        """One forward of a tree of drafts for every sequence: tokens[i] (ids) of sequence i, the first the last one it chose, the others drafts behind parents[i][j], an earlier one's number (the
        first's: -1).  Every node's next token is sampled from its logits with u [number of all nodes] (None: the largest), and the path of the drafts that are what was sampled
        stays in the cache (weights of drafts are not summed: their positions begin without any).  Returns per sequence the tokens behind the first, the last of them not in the cache yet: what decode would have given, one by one, with the u of the nodes on the path."""
        with torch.cuda.stream(stream):
            return self._decode_drafts(tokens, parents, temperature, top_k, top_p, min_p, u)

    def _decode_drafts(self, tokens, parents, temperature, top_k, top_p, min_p, u):
        run, n, rows = self.run, len(self.pages), [len(t) for t in tokens]
        if len(tokens) != n or len(parents) != n or any(len(p) != r for p, r in zip(parents, rows)) or not n or min(rows) < 1:
            raise ValueError(f"trees of {rows} nodes for {n} sequences, parents of {[len(p) for p in parents]}")
        if any(p >= i or p < 0 for tree in parents for i, p in enumerate(tree) if i):
            raise ValueError("a draft's parent is an earlier node of its tree")
        total = sum(rows)
        if u is not None and u.shape != (total,):
            raise ValueError(f"u is {list(u.shape)}, wanted [{total}]")
        held = self._grown((self.pages, self.length, self.free), list(range(n)), rows)
        batch = self._batch(held, list(range(n)), rows)
        parent, ids = self._int([p for tree in parents for p in tree]), self._int([x for tree in tokens for x in tree])
        seen, place = torch.empty(total, -(-max(rows) // 32), dtype=torch.int32, device=self.device), torch.empty(total, dtype=torch.int32, device=self.device)
        vb.vla_paged_tree(self.cache, batch, parent, seen, place)
        depth = place - torch.repeat_interleave(self._int([l - r for l, r in zip(held[1], rows)]), self._int(rows), output_size=total)
        logits = self._run_rows(held, list(range(n)), rows, ids, None, self.shared_len, depth=depth, seen=seen)
        every = lambda v, dtype: torch.full((total,), v, dtype=dtype, device=self.device)
        bins = torch.empty(total, dtype=torch.int32, device=self.device)
        vb.vla_sample_logits(logits, bins, every(temperature, torch.float32), every(top_k, torch.int32), every(top_p, torch.float32), every(min_p, torch.float32), u, None, None, None,
                             self._buf("ws_sample", vb.vla_sample_logits_workspace_bytes(total, vb.VLA_N_BINS)))
        chosen = torch.where(bins >= 0, bins + (run.shape.vocab - vb.VLA_N_BINS), -1).to(torch.int32)
        path, count = torch.empty(n, max(rows), dtype=torch.int32, device=self.device), torch.empty(n, dtype=torch.int32, device=self.device)
        following, new_len = torch.empty_like(count), torch.empty_like(count)
        vb.vla_paged_accept(self.cache, run.shape.n_layers, self.layer_stride, batch, parent, ids, chosen, path, count, following, new_len)
        if self.mass is not None:
            mass = self._room(n, max(held[1]))
            mass.masked_fill_(torch.arange(mass.shape[3], device=self.device) >= self._int(self.length)[:, None, None], 0.0)
        path, following, new_len = path.tolist(), following.tolist(), new_len.tolist()
        self._hold((held[0], new_len, held[2]))
        return [[tokens[i][j] for j in path[i][1:] if j >= 0] + [following[i]] for i in range(n)]

    def _decode(self, logits, n_tokens, temperature, top_k, top_p, min_p, u, select=0):
        run, n, dev = self.run, logits.shape[0], self.run.device
        if n != len(self.pages) or n_tokens < 1:
            raise ValueError(f"{n_tokens} tokens from logits of {n} sequences: there are {len(self.pages)}")
        if u is not None and (u.dim() != 2 or u.shape[0] < n_tokens or u.shape[1] != n):
            raise ValueError(f"u is {list(u.shape)}, wanted [{n_tokens}, {n}]")
        most = -(-max(self._grown((self.pages, self.length, self.free), list(range(n)), [n_tokens - 1] * n)[1]) // self.page_size)          # (the pages of all steps, before the first)
        if select and n_tokens > 1 and most > vb.VLA_SELECT_PAGES:
            raise ValueError(f"{most} pages of a sequence to select from, at most {vb.VLA_SELECT_PAGES}")
        every = lambda v, dtype: torch.full((n,), v, dtype=dtype, device=dev)
        t, k, p, least = every(temperature, torch.float32), every(top_k, torch.int32), every(top_p, torch.float32), every(min_p, torch.float32)
        if select < 0 or (select and self.weigh):
            raise ValueError(f"select {select}: not negative, and not where weights are summed")
        ws = self._buf("ws_sample", vb.vla_sample_logits_workspace_bytes(n, vb.VLA_N_BINS))
        bounds = self._all_bounds() if select and n_tokens > 1 else None
        out = [[], [], [], []]
        for j in range(n_tokens):
            bins, logp, kept = (torch.empty(n, dtype=d, device=dev) for d in (torch.int32, torch.float32, torch.float32))
            vb.vla_sample_logits(logits, bins, t, k, p, least, None if u is None else u[j].contiguous(), logp, kept, None, ws)
            for o, x in zip(out, (bins, logp, kept, logits)):
                o.append(x)
            if j + 1 < n_tokens:
                _, logits, _ = self._forward(list(range(n)), bins + (run.shape.vocab - vb.VLA_N_BINS), [1] * n, shared_len=self.shared_len, select=select, bounds=bounds)
        return tuple(torch.stack(o, 1) for o in out)


class PipelinedRollout:
    """Rollout epoch with fine-grained pipelining on one GPU (section IV-A, hybrid mode, figure with
    k = 2): the environments are split into k sub-batches; while the simulator steps one sub-batch, the
    policy generates the actions of the next.  Each sub-batch has its own stream, KV buffer and
    workspace.  The simulator is the caller's: ``sim_step(j, t, bins_host)`` is called on a worker thread
    once the actions of sub-batch j at step t are on the host, and returns when that sub-batch's next
    observation exists (here the observation tensors stay the same; what the simulator computes is
    outside this library).  k = 1 is the collocated schedule: generation and simulation alternate."""

    def __init__(self, run: Rollout, k: int):
        import concurrent.futures
        self.run, self.k = run, k
        self.streams = [torch.cuda.Stream(device=run.device) for _ in range(k)]      # default priority
        self.pool = concurrent.futures.ThreadPoolExecutor(max_workers=k)

    def epoch(self, obs, m_chunks: int, S: int, A: int, sim_step, mode=0, slot_embed=None, temperature=1.0,
              gumbel=None):
        """obs[j] = (patch, ids) of sub-batch j (device tensors); gumbel[j] its noise or None.
        Returns (outputs, log): outputs[t][j] = (bins, logp, entropy) device tensors, log a list of
        (event, j, t, time) host timestamps in seconds from the start."""
        import time
        torch.cuda.synchronize(self.run.device)      # inputs made on other streams are complete
        t0 = time.perf_counter()
        log = []
        gen_done = None                              # the Generation side takes one sub-batch at a time
        pending = [None] * self.k
        outputs = []
        host_bins = [torch.empty(obs[j][0].shape[0], A, dtype=torch.int32).pin_memory() for j in range(self.k)]

        def simulate(j, t, ready):
            ready.synchronize()                      # the actions of (j, t) are on the host
            log.append(("actions", j, t, time.perf_counter() - t0))
            sim_step(j, t, host_bins[j])
            log.append(("observation", j, t, time.perf_counter() - t0))

        for t in range(m_chunks):
            row = []
            for j in range(self.k):
                if pending[j] is not None:
                    pending[j].result()              # o_t of sub-batch j exists
                patch, ids = obs[j]
                st = self.streams[j]
                log.append(("generate", j, t, time.perf_counter() - t0))
                with torch.cuda.stream(st):
                    if gen_done is not None:
                        st.wait_event(gen_done)
                    h_last, _ = self.run.prefill(patch, ids, want_value=False, stream=st, lane=j)
                    bins, logp, ent, _ = self.run.decode(h_last, S, A, mode, slot_embed, temperature,
                                                         None if gumbel is None else gumbel[j], want_logits=False,
                                                         stream=st, lane=j)
                    host_bins[j].copy_(bins, non_blocking=True)
                    ready = torch.cuda.Event()
                    ready.record(st)
                    gen_done = ready
                row.append((bins, logp, ent))
                pending[j] = self.pool.submit(simulate, j, t, ready)
            outputs.append(row)
        for f in pending:
            if f is not None:
                f.result()
        return outputs, log, time.perf_counter() - t0

    def close(self):
        self.pool.shutdown(wait=True)
