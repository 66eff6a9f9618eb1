"""Thin decode-loop driver over the C-ABI calls: owns the device buffers (weight
arena, paged KV cache, per-row state, outputs, workspace) as torch tensors and
chains  hydra_draft_tree -> tree_verify_forward -> accept_greedy -> kv_compact.

No arithmetic of the method happens here; torch is used to allocate memory, to
copy results into a log, and to provide the stream.
"""
from __future__ import annotations

from typing import Callable, Dict, List, Optional, Sequence, Tuple

import torch

from . import binding as hb


def chain_parent(T: int) -> List[int]:
    return [-1] + list(range(T - 1))


class _Outputs:
    def __init__(self, ctx: hb.Hydra, B: int, d: int, V: int, dev, want_logits: bool):
        T, P = ctx.T, ctx.depth + 1
        i32, f32 = torch.int32, torch.float32
        self.tree_tokens = torch.zeros(B, T, dtype=i32, device=dev)
        self.hidden = torch.zeros(B, T, d, dtype=f32, device=dev)
        self.argmax = torch.zeros(B, T, dtype=i32, device=dev)
        self.margin = torch.zeros(B, T, dtype=f32, device=dev)
        self.logits = torch.zeros(B, T, V, dtype=f32, device=dev) if want_logits else None
        self.n_acc = torch.zeros(B, dtype=i32, device=dev)
        self.path = torch.zeros(B, P, dtype=i32, device=dev)
        self.next_root = torch.zeros(B, dtype=i32, device=dev)
        self.last_node = torch.zeros(B, dtype=i32, device=dev)
        self.kv_index = torch.zeros(B, P, 2, dtype=i32, device=dev)


class Session:
    """`shape` needs attributes d, NL, H, Dh, F, V, dtype ('f32'|'bf16'), K, mlp_layers, rms_eps,
    rope_theta, include_root_embedding.  `get_tensor(name)` returns the named weight as a
    device tensor in the model dtype (names as in the weight generator).

    cache_format 'int8' or 'e4m3' (bf16 models): whole pages of the base cache are held in 8 bits; a row keeps the
    few 16-bit pages of its last, incomplete page and of a step's tree nodes.
    pool_pages: the cache has that many pages for all rows together (B * max_len tokens have not to fit), which rows take
    as they grow, share after fork() and give back with free_rows(); defragment() moves the pages in use to the front.

    What a text of any length costs can be bounded (positions go on, up to max_len): window = W lets a token see the last W positions and the first
    `sinks`; budget = (keep, recent, slack) keeps about `keep` tokens per layer and head, the first `sinks`, the last `recent` and those that drew most
    attention so far; between steps and prompt chunks no row holds more than keep + slack.  A prompt's tokens all count, of a step its root, the one
    node that is sure to stay when the weights are added up: of n tokens that a step accepts n - 1 give none away and begin with none, so what is kept behind generated text depends on
    the tree and on acceptance and is not what decoding token by token would keep under the same budget (one node a step: it is).
    With pool_pages, pages that nobody sees any more go back to the pool.  A step under a budget that is captured into a graph cuts the rows over keep + slack / 2
    on every replay; not behind fork(), where a cut waits for the device."""

    def __init__(self, shape, parent: Sequence[int], B: int, max_len: int,
                 get_tensor: Callable[[str], torch.Tensor], device="cuda:0", prefill_chunk: int = 64,
                 page_perm_seed: Optional[int] = None, want_logits: bool = False, max_pos: Optional[int] = None,
                 cache_format: Optional[str] = None, pool_pages: Optional[int] = None, window: Optional[int] = None, sinks: int = 0,
                 budget: Optional[Tuple[int, int, int]] = None):
        if cache_format not in (None, "int8", "e4m3"):
            raise ValueError(f"cache_format {cache_format!r}: None (16 bits), 'int8' or 'e4m3'")
        if cache_format and shape.dtype != "bf16":
            raise ValueError("an 8-bit cache needs a bf16 model")
        if window is not None and budget is not None:
            raise ValueError("a window or a budget, not both")
        if (window is not None or budget is not None) and (cache_format or getattr(shape, "prefix", 0)):
            raise ValueError("windows and budgets are for caches in the model's own format, and for models without a prefix layer")
        if window is not None and window < 1 or sinks < 0 or (sinks and window is None and budget is None):
            raise ValueError("a window of at least 1; sinks >= 0, with a window or a budget")
        if budget is not None and (len(budget) != 3 or min(budget) < 0 or budget[0] < 1 or budget[1] + sinks > budget[0]):
            raise ValueError("budget: (keep, recent, slack) with sinks + recent <= keep")
        self.shape, self.B, self.dev = shape, B, torch.device(device)
        self.parent = list(parent)
        self.dtype_code = hb.HYDRA_BF16 if shape.dtype == "bf16" else hb.HYDRA_F32
        self.tdtype = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
        self.want_logits = want_logits
        self.prefill_chunk = min(prefill_chunk, 128)
        self._max_pos = max_pos or (max_len + 256)
        torch.cuda.set_device(self.dev)
        self._next_slot = 0
        self._ctx: Dict[str, hb.Hydra] = {}
        self._out: Dict[str, _Outputs] = {}
        self.main = self._make_ctx("main", self.parent)
        # weights
        self.arena = torch.empty(self.main.weights_bytes(), dtype=torch.uint8, device=self.dev)
        self._bind(self.main)
        self._load_weights(get_tensor)
        # KV cache
        self._T_max = T_max = max(len(self.parent), self.prefill_chunk)
        self.max_pages = (max_len + T_max + 15) // 16
        self.pool = pool_pages is not None
        self.n_pages = int(pool_pages) if self.pool else B * self.max_pages
        cache_dtype = torch.float16 if shape.dtype == "bf16" else torch.float32     # 2 or 4 bytes per element; content is private
        block = shape.H * 16 * shape.Dh
        i32 = dict(dtype=torch.int32, device=self.dev)
        if self.pool:
            self.page_table = torch.full((B, self.max_pages), -1, **i32)
            self.pages = hb.Pages(self.page_table, torch.zeros(self.n_pages, **i32))
            self._lists = torch.zeros(5, max(B, self.n_pages, 2), **i32)           # copies or moves, their (two) counts, forked rows, rows served
        else:
            if page_perm_seed is None:
                perm = torch.arange(self.n_pages, dtype=torch.int32)
            else:
                g = torch.Generator().manual_seed(page_perm_seed)
                perm = torch.randperm(self.n_pages, generator=g).to(torch.int32)
            self.page_table = perm.reshape(B, self.max_pages).contiguous().to(self.dev)
        self.kv8: Optional[hb.KV8] = None
        if cache_format is None:
            self.k_pages = torch.zeros(shape.NL * self.n_pages * block, dtype=cache_dtype, device=self.dev)
            self.v_pages = torch.zeros(shape.NL * self.n_pages * block, dtype=cache_dtype, device=self.dev)
            self.kv = hb.KV(self.k_pages, self.v_pages, self.page_table, self.n_pages, seq_len_hint=0)
        else:
            # 16-bit pages that a row can need at once: those of the slots 16 n .. 16 n + 14 + T, taken in turn; from a small pool of their
            # own (with one more per row for copies) where rows can be forked
            ring = (T_max + 14) // 16 + 1
            self.n_tail = B * (ring + (1 if self.pool else 0))
            self.k_pages = torch.zeros(shape.NL * self.n_tail * block, dtype=cache_dtype, device=self.dev)
            self.v_pages = torch.zeros(shape.NL * self.n_tail * block, dtype=cache_dtype, device=self.dev)
            if self.pool:
                tail_table = torch.full((B, self.max_pages), -1, **i32)
                self.tail_pages = hb.Pages(tail_table, torch.zeros(self.n_tail, **i32))
            else:
                tail_table = (torch.arange(B, **i32)[:, None] * ring + torch.arange(self.max_pages, **i32)[None, :] % ring).contiguous()
            self.kv = hb.KV(self.k_pages, self.v_pages, tail_table, self.n_tail, seq_len_hint=0)
            self.k_codes = torch.zeros(shape.NL * self.n_pages * block, dtype=torch.uint8, device=self.dev)
            self.v_codes = torch.zeros(shape.NL * self.n_pages * block, dtype=torch.uint8, device=self.dev)
            self.kv8 = hb.KV8(self.kv, self.k_codes, self.v_codes, torch.ones(shape.NL, self.n_pages, shape.H, 2, device=self.dev), self.page_table,
                              torch.zeros(B, **i32), self.n_pages, hb.KV8_INT8 if cache_format == "int8" else hb.KV8_E4M3)
        if self.pool:
            most = max(self.n_pages, self.kv.n_pages)
            self._pages_ws = torch.empty(hb.pages_workspace_bytes(B, most, self.max_pages), dtype=torch.uint8, device=self.dev)
        # part of the cache
        self.span: Optional[hb.KVSpan] = None
        self.budget = budget
        if window is not None or budget is not None:
            first = score = None
            if budget is not None:
                first = torch.zeros(B, **i32)
                score = torch.zeros(shape.NL, B, shape.H, 16 * self.max_pages, dtype=torch.float32, device=self.dev)
                self._kept = torch.zeros(shape.NL, B, shape.H, budget[0], **i32)
                self._evicted = torch.zeros(B, **i32)
            self.span = hb.KVSpan(self.kv, first=first, n_sinks=sinks, window=window or 0, score=score)
            self._growth = 0                          # tokens that a row can have taken since the last cut
            self._replays = False                     # whether a graph holds a step: replays make rows longer than host_len knows
            self._shared = False                      # rows may share pages
            if self.pool:
                self._lo = torch.zeros(B, **i32)
                self._dst = hb.Pages(torch.full((B, self.max_pages), -1, **i32), self.pages.ref)
        # state
        self.seq_len = torch.zeros(B, dtype=torch.int32, device=self.dev)
        self.h_last = torch.zeros(B, shape.d, dtype=torch.float32, device=self.dev)
        self.root = torch.zeros(B, dtype=torch.int32, device=self.dev)
        self.host_len = 0                     # host upper bound on seq_len (hint only)
        self._other_len = 0                   # the same of the rows that take no part in a prompt
        # the bound is tightened without stalling: every few steps seq_len is copied to pinned memory and picked
        # up once the copy has landed
        self._len_pinned = torch.zeros(B, dtype=torch.int32).pin_memory()
        self._len_event: Optional[torch.cuda.Event] = None
        self._growth_since_copy = 0
        self._steps_since_copy = 0
        self.ws = torch.empty(max(self.main.workspace_bytes(B), 256), dtype=torch.uint8, device=self.dev)
        # Hydra++ prefix attention: a one-layer context family of its own (weights, cache, length); it shares the
        # page table with the base cache (same slots, its own page storage)
        self.prefix = bool(getattr(shape, "prefix", 0))
        self._pctx: Dict[int, hb.Hydra] = {}
        if self.prefix:
            self._pnext_slot = 0
            first = self._prefix_ctx_new(self.main.depth + 1)
            self.parena = torch.empty(first.weights_bytes(), dtype=torch.uint8, device=self.dev)
            self._prefix_bind(first)
            for nm, kind in (("attn_norm", hb.W_ATTN_NORM), ("wq", hb.W_WQ), ("wk", hb.W_WK), ("wv", hb.W_WV), ("wo", hb.W_WO),
                             ("ffn_norm", hb.W_FFN_NORM), ("w_gate", hb.W_GATE), ("w_up", hb.W_UP), ("w_down", hb.W_DOWN)):
                first.load_tensor(kind, 0, 0, get_tensor(f"prefix.{nm}"))
            first.load_tensor(hb.W_FINAL_NORM, 0, 0, torch.ones(shape.d, dtype=self.tdtype, device=self.dev))   # never used; kept defined
            torch.cuda.synchronize()
            n_el1 = self.n_pages * block
            self.pk_pages = torch.zeros(n_el1, dtype=cache_dtype, device=self.dev)
            self.pv_pages = torch.zeros(n_el1, dtype=cache_dtype, device=self.dev)
            self.pkv = hb.KV(self.pk_pages, self.pv_pages, self.page_table, self.n_pages, seq_len_hint=0)
            self.pseq_len = torch.zeros(B, dtype=torch.int32, device=self.dev)

    # ---- contexts -----------------------------------------------------------
    def _make_ctx(self, name: str, parent: Sequence[int]) -> hb.Hydra:
        s = self.shape
        ctx = hb.Hydra(d=s.d, n_layers=s.NL, n_heads=s.H, head_dim=s.Dh, ffn=s.F, vocab=s.V, dtype=self.dtype_code,
                       rms_eps=s.rms_eps, rope_theta=s.rope_theta, max_pos=self._max_pos, n_draft_heads=s.K,
                       mlp_layers=s.mlp_layers, include_root_embedding=s.include_root_embedding, medusa=getattr(s, "medusa", 0),
                       parent=parent, max_batch=self.B)
        self._ctx[name] = ctx
        self._out[name] = _Outputs(ctx, self.B, s.d, s.V, self.dev, self.want_logits)
        return ctx

    def _bind(self, ctx: hb.Hydra) -> None:
        ctx.bind_weights(self.arena, self._next_slot)
        self._next_slot += 1

    def _check_nodes(self, T: int) -> None:
        """Behind an 8-bit cache the 16-bit pages are taken in turn: the nodes of a larger tree would overwrite each other."""
        if self.kv8 is not None and T > self._T_max:
            raise ValueError(f"an 8-bit cache of this session has 16-bit pages for trees of up to {self._T_max} nodes")

    def ctx(self, name: str) -> hb.Hydra:
        """'main', 'ar' (one-node tree) or 'chainN' (N-token causal chunk), created on demand."""
        if name not in self._ctx:
            parent = [-1] if name == "ar" else chain_parent(int(name[5:]))
            self._check_nodes(len(parent))
            c = self._make_ctx(name, parent)
            self._bind(c)
            need = c.workspace_bytes(self.B)
            if need > self.ws.numel():
                torch.cuda.synchronize()
                self.ws = torch.empty(need, dtype=torch.uint8, device=self.dev)
        return self._ctx[name]

    def add_tree(self, name: str, parent: Sequence[int]) -> hb.Hydra:
        """A further decode context with its own candidate tree on the same weights and cache (the weight arena has
        room for 16 contexts in all)."""
        if name in self._ctx:
            raise ValueError(f"context {name!r} exists")
        self._check_nodes(len(parent))
        c = self._make_ctx(name, list(parent))
        self._bind(c)
        need = c.workspace_bytes(self.B)
        if need > self.ws.numel():
            torch.cuda.synchronize()
            self.ws = torch.empty(need, dtype=torch.uint8, device=self.dev)
        return c

    # ---- prefix-attention contexts (one per chain length) --------------------------
    def _prefix_ctx_new(self, P: int) -> hb.Hydra:
        s = self.shape
        c = hb.Hydra(d=s.d, n_layers=1, n_heads=s.H, head_dim=s.Dh, ffn=s.F, vocab=32, dtype=self.dtype_code,
                     rms_eps=s.rms_eps, rope_theta=s.rope_theta, max_pos=self._max_pos, n_draft_heads=0,
                     mlp_layers=1, include_root_embedding=1, parent=chain_parent(P), max_batch=self.B)
        self._pctx[P] = c
        return c

    def _prefix_bind(self, c: hb.Hydra) -> None:
        c.bind_weights(self.parena, self._pnext_slot)
        self._pnext_slot += 1
        need = c.workspace_bytes(self.B)
        if need > self.ws.numel():
            torch.cuda.synchronize()
            self.ws = torch.empty(need, dtype=torch.uint8, device=self.dev)

    def prefix_ctx(self, P: int) -> hb.Hydra:
        if P not in self._pctx:
            self._prefix_bind(self._prefix_ctx_new(P))
        return self._pctx[P]

    def prefix_attention(self, name: str = "main", rows: Optional[int] = None) -> None:
        """Feeds the accepted tokens' hidden states of context `name` to the prefix layer; h_last becomes its output (the first `rows` rows)."""
        c, o = self._ctx[name], self._out[name]
        P = o.path.shape[1]
        self.pkv.seq_len_hint = self.host_len
        self.prefix_ctx(P).hydra_prefix_attention(rows or self.B, self.ws, o.hidden, c.T, o.path, o.n_acc, self.pseq_len, self.pkv, self.h_last)

    def out(self, name: str = "main") -> _Outputs:
        return self._out[name]

    def _load_weights(self, get) -> None:
        s, m = self.shape, self.main
        m.load_tensor(hb.W_EMBED, 0, 0, get("embed"))
        m.load_tensor(hb.W_LM_HEAD, 0, 0, get("lm_head"))
        m.load_tensor(hb.W_FINAL_NORM, 0, 0, get("final_norm"))
        per_layer = (("attn_norm", hb.W_ATTN_NORM), ("wq", hb.W_WQ), ("wk", hb.W_WK), ("wv", hb.W_WV), ("wo", hb.W_WO),
                     ("ffn_norm", hb.W_FFN_NORM), ("w_gate", hb.W_GATE), ("w_up", hb.W_UP), ("w_down", hb.W_DOWN))
        for l in range(s.NL):
            for nm, kind in per_layer:
                m.load_tensor(kind, l, 0, get(f"layers.{l}.{nm}"))
            torch.cuda.synchronize()          # sources may be freed by the provider
        for i in range(1, s.K + 1):
            m.load_tensor(hb.W_HEAD_W1, i, 0, get(f"heads.{i}.w1"))
            m.load_tensor(hb.W_HEAD_B1, i, 0, get(f"heads.{i}.b1"))
            for j in range(2, s.mlp_layers + 1):
                m.load_tensor(hb.W_HEAD_WL, i, j, get(f"heads.{i}.w{j}"))
                m.load_tensor(hb.W_HEAD_BL, i, j, get(f"heads.{i}.b{j}"))
            m.load_tensor(hb.W_HEAD_WOUT, i, 0, get(f"heads.{i}.wout"))
            torch.cuda.synchronize()

    # ---- steps ----------------------------------------------------------------
    def _hint(self, T: int) -> None:
        if self.pool and self.host_len + T > min(self.max_pages * 16, self._max_pos):
            self.sync_len()                           # rows may have been freed since: only the real lengths are refused
        self.kv.seq_len_hint = self.host_len
        if self.span is not None:
            self.span.span_hint = self._most_held()

    def _most_held(self) -> int:
        """Host bound on the tokens that a row holds (0: nothing is known to hold any)."""
        held = max(self.host_len, self._other_len)
        if self.budget is not None:
            keep, _, slack = self.budget
            most = keep + slack // 2 + self._growth
            held = most if self._replays else min(held, most)
        return held

    def reset(self) -> None:
        self.seq_len.zero_(); self.h_last.zero_(); self.root.zero_()
        if self.prefix:
            self.pseq_len.zero_()
        if self.kv8 is not None:
            self.kv8.n_sealed.zero_()
        if self.budget is not None:
            self.span.first.zero_()
            self.span.score.zero_()
        if self.span is not None:
            self._growth, self._shared = 0, False
        if self.pool:
            for p in self._pools():
                p.page_table.fill_(-1)
                p.ref.zero_()
        self.host_len = 0
        self._len_event = None

    # ---- the cache behind a forward pass, in 16 or 8 bits ------------------------
    def _forward(self, c: hb.Hydra, o: _Outputs, B: int, prompt: bool = False) -> None:
        args = (o.tree_tokens, self.seq_len[:B])
        out = (o.hidden, o.argmax, o.margin, o.logits)
        if self.span is not None:
            self.span.n_scored = c.T if prompt else 1
            c.tree_verify_forward_span(B, self.ws, *args, self.span, *out)
        elif self.kv8 is None:
            c.tree_verify_forward(B, self.ws, *args, self.kv, *out)
        else:
            c.tree_verify_forward_kv8(B, self.ws, *args, self.kv8, *out)

    def _keep_accepted(self, c: hb.Hydra, o: _Outputs, B: int, h_last: torch.Tensor, root: torch.Tensor) -> None:
        # (no hydra_score_compact: a prompt's path is the identity, and the root of a step sees no other node, so their sums all begin at 0)
        if self.budget is not None:
            self._growth += c.depth + 1               # first: whatever is broken off behind this is not forgotten
        c.kv_compact(B, o.n_acc, o.path, o.next_root, o.last_node, o.hidden, self.kv, self.seq_len, h_last, root, o.kv_index)
        if self.kv8 is not None:
            c.hydra_kv8_seal(B, self.seq_len, self.kv8)

    def _trim(self) -> None:
        """Rows over the budget are cut, once in a while: a cut leaves at most keep + slack / 2 tokens, and the next one comes before a row can have taken
        the other half.  A graph gets the cut with each step, which then cuts the rows over keep + slack / 2 on every replay."""
        if self.budget is None:
            return
        keep, recent, slack = self.budget
        captures = torch.cuda.is_current_stream_capturing()
        if captures and self.pool and self._shared:
            raise RuntimeError("the cut of rows that may share pages waits for the device: such a step cannot be captured")
        self._replays |= captures
        most = max(self.host_len, self._other_len)
        if not captures and (self._growth <= slack - slack // 2 or (most <= keep + slack // 2 and not self._replays)):
            return
        self.span.span_hint = keep + slack + self._growth if self._replays else most
        if self.pool and self._shared:
            self._cut_shared(keep, recent, slack // 2)
        else:
            self.main.hydra_kv_evict(self.B, self.seq_len, self.span, keep, recent, slack // 2, self._kept, self._evicted)
        if not captures:                              # (nothing has run: what a row may have taken stays counted)
            self._growth = 0

    def _cut_shared(self, keep: int, recent: int, spare: int) -> None:
        """The cut of rows that may share pages (waits for the device): those that do go to pages of their own, and what they held goes back where no other row has it; the others
        are cut where they lie.  A row that a call must leave alone is shown to it with no tokens (first = seq_len)."""
        m, B, span, first = self.main, self.B, self.span, self.span.first
        at = torch.arange(0, 16 * self.max_pages, 16, dtype=torch.int32, device=self.dev)
        held = (self.page_table >= 0) & (at + 16 > first[:, None]) & (at < self.seq_len[:, None])
        refs = self.pages.ref[self.page_table.clamp(0, self.n_pages - 1).long()]
        moves = (self.seq_len - first > keep + spare) & (held & (refs > 1)).any(dim=1)
        some, self._shared = torch.stack([moves.any(), (self.pages.ref > 1).any()]).tolist()
        own = torch.where(moves, self.seq_len, first)

        def cut(of: torch.Tensor, dst: Optional[torch.Tensor]) -> None:
            m.hydra_kv_evict(B, self.seq_len, hb.KVSpan(span.kv, of, span.n_sinks, 0, span.span_hint, span.score), keep, recent, spare, self._kept, self._evicted, dst_table=dst)

        cut(own, None)
        first.copy_(torch.where(moves, first, own))
        if not some:
            return
        here = self._evicted.clone()
        self._drop_scratch()                          # with what those rows have left
        zero = torch.zeros_like(self.seq_len)
        whole = zero + 16 * self.max_pages
        m.hydra_pages_reserve(B, self._pages_ws, self._dst, torch.where(moves, self.seq_len - keep, zero), torch.where(moves, self.seq_len, zero), 0, self._lists[4])
        if not bool(self._lists[4][:B].all()):
            m.hydra_pages_release(B, self._dst, None, zero)
            raise RuntimeError(f"the pool of {self.n_pages} pages is exhausted: no room for the kept tokens of rows that share pages")
        own = torch.where(moves, first, self.seq_len)
        cut(own, self._dst.page_table)
        done = self._evicted > 0
        first.copy_(torch.where(done, own, first))
        m.hydra_pages_release(B, self.pages, None, torch.where(done, zero, whole))
        m.hydra_pages_release(B, self._dst, None, torch.where(done, whole, zero))        # of rows that had to stay whole
        self.page_table.copy_(torch.where(done[:, None], self._dst.page_table, self.page_table))
        self._dst.page_table.fill_(-1)
        self._evicted += here

    def _incomplete(self) -> torch.Tensor:
        """The 16-bit page of every row that its next token goes to (any page where the row holds none there)."""
        at = (self.seq_len // 16).clamp(max=self.max_pages - 1).long()
        return self.kv.page_table.gather(1, at[:, None])[:, 0].clamp(min=0).long()

    def _mark(self):
        """What _back_to needs to return to the text as it is now.  Behind an 8-bit cache 16-bit pages are taken again as the text grows:
        every row's incomplete one is kept apart.  Sealed pages are never written again."""
        mark = [[t.clone() for t in (self.seq_len, self.h_last, self.root)], self.host_len]
        if self.kv8 is not None:
            pages = self._incomplete()
            mark += [self.kv8.n_sealed.clone()] + [t.view(self.shape.NL, self.n_tail, -1)[:, pages] for t in (self.k_pages, self.v_pages)]
        return mark

    def _back_to(self, mark) -> None:
        for t, kept in zip((self.seq_len, self.h_last, self.root), mark[0]):
            t.copy_(kept)
        self.host_len = mark[1]
        if self.kv8 is None:
            return
        self.kv8.n_sealed.copy_(mark[2])
        if self.pool:
            lo = self.kv8.n_sealed * 16
            self.main.hydra_pages_release(self.B, self.tail_pages, lo, self.seq_len)
            self.main.hydra_pages_reserve(self.B, self._pages_ws, self.tail_pages, lo, self.seq_len, 0)
        rows = (self.seq_len % 16).nonzero()[:, 0]
        pages = self._incomplete()[rows]
        for t, kept in zip((self.k_pages, self.v_pages), mark[3:]):
            t.view(self.shape.NL, self.n_tail, -1)[:, pages] = kept[:, rows]

    # ---- pages ------------------------------------------------------------------
    def _pools(self) -> List[hb.Pages]:
        return [self.pages] if self.kv8 is None else [self.pages, self.tail_pages]

    def _need_pool(self) -> None:
        if not self.pool:
            raise ValueError("rows of this session have pages of their own: create the Session with pool_pages")

    def _drop_scratch(self) -> None:
        """The pages behind every row's text go back."""
        if self.span is not None:
            self.main.hydra_pages_release_span(self.B, self.pages, self.seq_len, self.span)
            return
        for p in self._pools():
            self.main.hydra_pages_release(self.B, p, None, self.seq_len)

    def _reserve(self, T: int, B: int) -> None:
        """Pages for T more slots of the first B rows.  Waits for the device only where the pool might be too small: a row holds no
        pages but those of its text and of the nodes of one tree or chunk, so whatever shortens a text gives pages back too."""
        if not self.pool:
            return
        ok = self._lists[4]
        lo = None
        if self.span is not None:                     # what no node sees any more goes back first, and stays without pages
            lo = self._lo                             # (of every row: a cut empties pages of those too that take no part in a prompt)
            self.main.hydra_pages_release_span(self.B, self.pages, self.seq_len, self.span, lo)
        self.main.hydra_pages_reserve(B, self._pages_ws, self.pages, lo, self.seq_len, T, ok)
        if self.kv8 is not None:
            # never short of pages: no tree has more than _T_max nodes (_check_nodes), so a row holds at most a ring of them, and fork() takes
            # one more for each row
            lo = self.kv8.n_sealed * 16
            self.main.hydra_pages_release(B, self.tail_pages, lo, self.seq_len)
            self.main.hydra_pages_reserve(B, self._pages_ws, self.tail_pages, lo, self.seq_len, T)
        # a row may hold pages that the nodes of a larger tree than this one needed
        most, held = max(c.T for c in self._ctx.values()), max(self.host_len, self._other_len)
        if self.span is not None:                     # with the ends of two stretches, sinks and the rest, inside pages
            held = min(held, self.span.window + self.span.n_sinks if self.span.window else self._most_held()) + 45
        if self.B * ((held + most + 15) // 16) > self.n_pages and not bool(ok[:B].all()):
            raise RuntimeError(f"the pool of {self.n_pages} pages is exhausted")

    def fork(self, src_rows: Sequence[int]) -> None:
        """Row b becomes a copy of row src_rows[b] as it is now (b or -1: stays).  Whole pages are shared; only the last, incomplete page
        is copied.  For samples of one prompt, or beams that change places."""
        self._need_pool()
        if len(src_rows) != self.B or any(r < -1 or r >= self.B or r != int(r) for r in src_rows):
            raise ValueError(f"fork: {self.B} rows of [-1, {self.B})")
        B, m = self.B, self.main
        want = torch.tensor([b if r < 0 else r for b, r in enumerate(src_rows)], dtype=torch.int32, device=self.dev)
        src, dst, forked = self._lists[0], self._lists[1], self._lists[3]
        self._drop_scratch()                          # what the last step left goes back first
        m.hydra_pages_fork(B, self._pages_ws, self.pages, want, self.seq_len, src, dst, forked)
        if not torch.equal(forked[:B], want):
            got = forked[:B].clone()
            self._take_rows(got, src, dst)
            raise RuntimeError(f"the pool of {self.n_pages} pages is exhausted: rows {(got != want).nonzero()[:, 0].tolist()} stay as they were")
        self._take_rows(forked[:B].clone(), src, dst)

    def _take_rows(self, rows: torch.Tensor, src: torch.Tensor, dst: torch.Tensor) -> None:
        """Contents and state of rows that the tables say are copies now."""
        B, m = self.B, self.main
        if self.kv8 is None:
            m.hydra_kv_copy_pages(self.kv, B, src, dst)
        if self.prefix:
            self.prefix_ctx(self.main.depth + 1).hydra_kv_copy_pages(self.pkv, B, src, dst)
        if self.kv8 is not None:
            m.hydra_pages_fork(B, self._pages_ws, self.tail_pages, rows, self.seq_len, src, dst, self._lists[3])
            m.hydra_kv_copy_pages(self.kv, B, src, dst)
        state = [self.seq_len, self.h_last, self.root] + ([self.pseq_len] if self.prefix else []) + ([self.kv8.n_sealed] if self.kv8 is not None else [])
        if self.span is not None:
            self._shared = True
        if self.budget is not None:
            state.append(self.span.first)
            for layer in self.span.score:
                layer.copy_(layer[rows.long()])
        for t in state:
            t.copy_(t[rows.long()])
        self._len_event = None                        # a length on its way to the host may be another row's

    def free_rows(self, rows: Sequence[int]) -> None:
        """The rows' text ends: they start again from nothing, and their pages (where no other row shares them) are free.
        A step adds to such a row as to any other: free it again before it takes its next prompt."""
        self._need_pool()
        if any(r != int(r) or r < 0 or r >= self.B for r in rows):
            raise ValueError(f"free_rows: rows of [0, {self.B})")
        at = torch.tensor(list(rows), dtype=torch.int64, device=self.dev)
        for t in [self.seq_len, self.h_last, self.root] + ([self.pseq_len] if self.prefix else []) + ([self.kv8.n_sealed] if self.kv8 is not None else []):
            t.index_fill_(0, at, 0)
        if self.budget is not None:
            self.span.first.index_fill_(0, at, 0)
            self.span.score.index_fill_(1, at, 0)
        self._drop_scratch()

    def defragment(self) -> int:
        """Gives back what no text needs, moves the pages in use to the front of the pool and returns how many they are (waits for the device)."""
        self._need_pool()
        m, (src, dst, counts) = self.main, self._lists[:3]
        self._drop_scratch()
        m.hydra_pages_compact(self.B, self._pages_ws, self.pages, src, dst, counts)
        if self.kv8 is None:
            m.hydra_kv_copy_pages(self.kv, self.n_pages, src, dst, counts)
        else:
            m.hydra_kv8_copy_pages(self.kv8, self.n_pages, src, dst, counts)
        if self.prefix:
            self.prefix_ctx(m.depth + 1).hydra_kv_copy_pages(self.pkv, self.n_pages, src, dst, counts)
        return int(counts[1])

    def prefill(self, prompts: torch.Tensor, behind_chunk: Optional[Callable[[str, int, int], None]] = None) -> None:
        """prompts: int32 [B, L] (same length for every row; with pool_pages also fewer rows, the first ones).  Causal chunks through
        tree_verify_forward with a chain tree; the state update is kv_compact with the
        identity path.  Where an exception breaks the prompt off, seq_len, h_last and root are those behind the last chunk that was
        computed whole (behind the text in front of the prompt if there is none).  behind_chunk(context, position, tokens) is called when a chunk's outputs are
        there, which then all chunks have.  With a budget, what a chunk that was broken off added to the weights of the tokens in front of it stays."""
        B, L = prompts.shape
        assert B == self.B or (self.pool and B < self.B)
        prompts = prompts.to(self.dev, torch.int32)
        chunks = [min(self.prefill_chunk, L - pos) for pos in range(0, L, self.prefill_chunk)]
        # A chunk whose outputs a later chunk of the same length writes again ends behind the decoder layers: no final norm, LM head and
        # argmax, whose results nobody can read once the call is over.  Not where the prefix layer reads every chunk's hidden states, and not where the prompt
        # does not fit (the chunks in front of the one that is refused then keep their outputs and the state behind them).
        room = min(self.max_pages * 16, self._max_pos)
        if self.pool and self.host_len + L > room:    # rows may have been freed since, and the longest one may take no part
            lens = self.seq_len.tolist()
            self._other_len = max(lens[B:], default=0)
            self._set_len(max(lens[:B]))
        # Nor where a broken prompt could not go back, because what was cut or given back meanwhile is gone.
        layers_only = not self.prefix and self.host_len + L <= room and behind_chunk is None and self.budget is None and not (self.span is not None and self.pool)
        last = {n: i for i, n in enumerate(chunks)}
        pos = 0
        behind = None                                 # the text behind the last chunk that h_last and root know of, if others followed
        try:
            for i, n in enumerate(chunks):
                name = f"chain{n}"
                c = self.ctx(name)
                o = self._out[name]
                o.tree_tokens[:B].copy_(prompts[:, pos:pos + n])
                self._hint(n)
                self._reserve(n, B)
                if i == chunks.index(n):              # the same for every chunk of this length
                    o.n_acc.fill_(n)
                    o.path.copy_(torch.arange(n, dtype=torch.int32, device=self.dev).expand(self.B, n))
                    o.last_node.fill_(n - 1)
                h_last, root = self.h_last, self.root
                if layers_only and i < last[n]:
                    if behind is None:
                        behind = self._mark()
                    h_last, root = torch.empty_like(h_last), torch.empty_like(root)       # of outputs that are not written
                    if self.span is not None:
                        c.hydra_prefill_chunk_span(B, self.ws, o.tree_tokens, self.seq_len, self.span)
                    elif self.kv8 is None:
                        c.hydra_prefill_chunk(B, self.ws, o.tree_tokens, self.seq_len, self.kv)
                    else:
                        c.hydra_prefill_chunk_kv8(B, self.ws, o.tree_tokens, self.seq_len, self.kv8)
                else:
                    self._forward(c, o, B, prompt=True)
                    o.next_root.copy_(o.argmax[:, n - 1])
                    if behind_chunk is not None:
                        behind_chunk(name, pos, n)
                self._keep_accepted(c, o, B, h_last, root)
                if h_last is self.h_last:
                    behind = None
                if self.prefix:
                    self.prefix_attention(name, B)    # hint: still the length before this chunk
                pos += n
                self.host_len += n
                self._growth_since_copy += n          # a length on its way to the host was read before these
                self._trim()
        except BaseException:
            if behind is not None:                    # broken off: back to the text that h_last and root belong to
                self._back_to(behind)
            elif self.kv8 is not None:                # a whole chunk may have been broken off between its compaction and its seal
                self.main.hydra_kv8_seal(self.B, self.seq_len, self.kv8)
            if self.pool:                             # what _reserve goes by: no row holds more than its text and one step need
                self._drop_scratch()
            self.sync_len()
            raise
        finally:
            self.host_len, self._other_len = max(self.host_len, self._other_len), 0

    def draft(self, name: str = "main") -> None:
        c, o = self.ctx(name), self._out[name]
        c.hydra_draft_tree(self.B, self.ws, self.h_last, self.root, o.tree_tokens)

    def verify(self, name: str = "main") -> None:
        c, o = self.ctx(name), self._out[name]
        self._hint(c.T)
        self._reserve(c.T, self.B)
        self._forward(c, o, self.B)

    def accept(self, name: str = "main") -> None:
        c, o = self.ctx(name), self._out[name]
        c.accept_greedy(self.B, o.tree_tokens, o.argmax, o.n_acc, o.path, o.next_root, o.last_node)

    def accept_typical(self, tau: float, eps: float, alpha: float, u: Optional[torch.Tensor] = None, name: str = "main") -> None:
        """Typical acceptance instead of greedy acceptance; needs the session to keep logits (want_logits=True)."""
        c, o = self.ctx(name), self._out[name]
        if o.logits is None:
            raise ValueError("typical acceptance needs the logits: create the Session with want_logits=True")
        c.accept_typical(self.B, self.ws, o.tree_tokens, o.logits, tau, eps, alpha, u, o.n_acc, o.path, o.next_root, o.last_node)

    def logprobs(self, tokens: Optional[torch.Tensor] = None, tau: float = 1.0, k: int = 0, name: str = "main", rows: Optional[int] = None) -> Dict[str, torch.Tensor]:
        """Of the last forward pass through context `name` (a session that keeps logits): the entropy of every node's distribution, the log probability and rank of
        tokens [B, T] int32 (-1: none), and the k most likely tokens with theirs.  The first `rows` rows."""
        c, o = self.ctx(name), self._out[name]
        if o.logits is None:
            raise ValueError("log probabilities need the logits: create the Session with want_logits=True")
        B = rows or self.B
        f32, i32 = dict(dtype=torch.float32, device=self.dev), dict(dtype=torch.int32, device=self.dev)
        out = {"entropy": torch.empty(B, c.T, **f32)}
        if tokens is not None:
            if tuple(tokens.shape) != (B, c.T):
                raise ValueError(f"tokens: expected [{B}, {c.T}], got {tuple(tokens.shape)}")
            tokens = tokens.to(self.dev, torch.int32).contiguous()
            out |= {"logprob": torch.empty(B, c.T, **f32), "rank": torch.empty(B, c.T, **i32)}
        if k:
            out |= {"top_ids": torch.empty(B, c.T, k, **i32), "top_logprobs": torch.empty(B, c.T, k, **f32)}
        c.hydra_token_logprobs(B, self.ws, o.logits, tokens, tau, k, **out)
        return out

    def prompt_logprobs(self, prompts: torch.Tensor, tau: float = 1.0, k: int = 0) -> Dict[str, torch.Tensor]:
        """prefill(prompts), and what the model thought of them: entry i of a row is about the token behind prompt token i (behind the last one: none given).
        The mean of -logprob over a text says what a window, a budget or an 8-bit cache costs."""
        B, L = prompts.shape
        if not L or not self.want_logits:
            raise ValueError("log probabilities need a prompt, and the logits: create the Session with want_logits=True")
        parts: List[Dict[str, torch.Tensor]] = []
        given = torch.cat([prompts[:, 1:].to(self.dev, torch.int32), torch.full((B, 1), -1, dtype=torch.int32, device=self.dev)], dim=1)
        self.prefill(prompts, lambda name, pos, n: parts.append(self.logprobs(given[:, pos:pos + n], tau, k, name, B)))
        return {key: torch.cat([p[key] for p in parts], dim=1) for key in parts[0]}

    def compact(self, name: str = "main") -> None:
        c, o = self.ctx(name), self._out[name]
        self._hint(c.T)
        self._keep_accepted(c, o, self.B, self.h_last, self.root)
        self.host_len += c.depth + 1          # upper bound; the device holds the exact value
        self._growth_since_copy += c.depth + 1
        self._trim()

    def step(self, name: str = "main", hook=None, typical=None) -> None:
        """One speculative step of every row.  `hook(outputs)` may edit tree_tokens between
        draft and verify (scripted-acceptance experiments).  typical = (tau, eps, alpha, u): the accepted path
        and the next root come from accept_typical (u: device [B] uniform numbers or None) instead of accept_greedy."""
        self._refresh_bound()
        self.draft(name)
        if hook is not None:
            hook(self._out[name])
        self.verify(name)
        if typical is None:
            self.accept(name)
        else:
            self.accept_typical(typical[0], typical[1], typical[2], typical[3], name)
        pre = self.host_len
        self.compact(name)
        if self.prefix:
            post, self.host_len = self.host_len, pre          # the prefix cache is as long as the base cache was before compaction
            self.prefix_attention(name)
            self.host_len = post

    def _refresh_bound(self, every: int = 8) -> None:
        """Asynchronous tightening of the host bound on seq_len: no synchronisation, the value is used when it has arrived."""
        if self._len_event is not None and self._len_event.query():
            self.host_len = min(self.host_len, int(self._len_pinned.max()) + self._growth_since_copy)
            self._len_event = None
        self._steps_since_copy += 1
        if self._len_event is None and self._steps_since_copy >= every:
            self._len_pinned.copy_(self.seq_len, non_blocking=True)
            self._len_event = torch.cuda.Event()
            self._len_event.record()
            self._growth_since_copy = 0
            self._steps_since_copy = 0

    def sync_len(self) -> int:
        """Tighten the host bound from the device (synchronises)."""
        return self._set_len(int(self.seq_len.max().item()))

    def _set_len(self, longest: int) -> int:
        self.host_len = longest
        self._len_event = None
        self._steps_since_copy = 0
        return self.host_len

    def generate(self, n_new: int, name: str = "main", max_steps: Optional[int] = None):
        """Runs steps until every row has >= n_new tokens.  Returns (tokens per row, n_acc per step).

        fp32 models (a step is a few dozen launches of microseconds, as long on the host as on the GPU): while a further step is
        needed whatever the one before it accepts, it is enqueued before that one's result is waited for."""
        ctx = self.ctx(name)
        o = self._out[name]
        out = [[] for _ in range(self.B)]
        accs = []
        steps = 0
        # what a step is read back for goes to pinned memory in four copies behind one wait, instead of a wait per tensor
        src = (o.tree_tokens, o.path, o.n_acc, self.seq_len)
        host = [[torch.empty(t.shape, dtype=t.dtype, pin_memory=True) for t in src] for _ in range(2)]
        done = [torch.cuda.Event(), torch.cuda.Event()]
        ahead = 2 if self.dtype_code == hb.HYDRA_F32 else 1
        most = ctx.depth + 1                          # tokens that a step can add to a row
        unread: List[int] = []                        # buffers of the steps that are enqueued and not read back yet

        def wanted() -> bool:
            if min(len(t) for t in out) + len(unread) * most >= n_new or (max_steps is not None and steps >= max_steps):
                return False
            # the length is an upper bound while a result is outstanding: where only that bound is refused, the result comes first
            return not unread or (self.host_len + ctx.T <= self.max_pages * 16 and self.host_len + most <= self._max_pos)

        while True:
            while len(unread) < ahead and wanted():
                k = steps % 2
                self.step(name)
                for h, t in zip(host[k], src):
                    h.copy_(t, non_blocking=True)
                done[k].record()
                unread.append(k)
                steps += 1
            if not unread:
                break
            k = unread.pop(0)
            done[k].synchronize()
            tt, pa, na, lens = (h.tolist() for h in host[k])
            for b in range(self.B):
                out[b] += [tt[b][pa[b][j]] for j in range(na[b])]
            accs.append(na)
            self._set_len(max(lens) + len(unread) * most)
        return [t[:n_new] for t in out], accs
