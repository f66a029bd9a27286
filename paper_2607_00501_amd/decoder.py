"""Host sequencing of the decode steps of a dense grouped-query-attention
decoder (the Llama 3.2 / Qwen3 layer) over the library's entry points
(BaseRT Sec. 3.2: a token is embedding, per layer norm -> q/k/v projections
-> RoPE and cache append -> attention -> output projection -> residual and
norm -> SwiGLU feed-forward, then the final norm, the LM head and sampling).

Every arithmetic step runs in the library's kernels; this module owns the
device buffers and issues the calls in order on one stream, with no host
synchronisation, so a step (or several) can be captured in a HIP graph and
the sampled token stays on the device for the next step's embedding.
"""

import math
from dataclasses import dataclass, replace
from typing import List, Optional

import torch

from . import binding as B


@dataclass
class DecoderConfig:
    hidden: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    inter: int
    vocab: int
    layers: int
    eps: float = 1e-6
    theta: float = 1e6
    # (factor, low_freq_factor, high_freq_factor, original_len): the Llama 3
    # long-context RoPE frequencies (None: plain theta^(-2i/D))
    rope_scaling: Optional[tuple] = None


@dataclass
class LayerWeights:
    wq: B.QWeight
    wk: B.QWeight
    wv: B.QWeight
    wo: B.QWeight
    wg: B.QWeight
    wu: B.QWeight
    wd: B.QWeight
    attn_norm: torch.Tensor   # fp16 [hidden]
    ffn_norm: torch.Tensor    # fp16 [hidden]
    q_norm: Optional[torch.Tensor] = None   # fp16 [head_dim]: per-head q/k RMSNorm (the Qwen3 layer)
    k_norm: Optional[torch.Tensor] = None


class DenseDecoder:
    """Buffers and call order of one decode step.  Weights: device-layout
    quantised projections, fp16 embedding table and norm weights.

    fused: the two RMSNorms of a layer run inside the GEMVs that read them
    (qmatmul_gemv_grouped_rmsnorm, qmatmul_gemv_swiglu_rmsnorm_f16; any
    weight format, hidden <= 4096), with the residual stream alternating between
    two buffers; otherwise each norm is a launch of its own.

    rope_rows_interleaved: W_q and W_k were quantised from rows in
    binding.rope_interleave_rows order; then (with fused) RoPE and the cache
    append run as the epilogue of the q/k/v GEMV
    (qmatmul_gemv_qkv_rmsnorm_rope): 5 launches per layer."""

    def __init__(self, cfg: DecoderConfig, emb: torch.Tensor, layers: List[LayerWeights], norm: torch.Tensor,
                 lm_head: B.QWeight, max_len: int, fused: bool = True, rope_rows_interleaved: bool = False,
                 max_chunk: int = 512):
        self.cfg, self.emb, self.layers, self.norm, self.lm_head = cfg, emb, layers, norm, lm_head
        self.max_len = max_len
        self.max_chunk = max_chunk          # rows of a prompt chunk (prefill)
        self._chunk = None
        dev = emb.device
        f32 = dict(dtype=torch.float32, device=dev)
        f16 = dict(dtype=torch.float16, device=dev)
        c = cfg
        qd, kvd = c.n_q_heads * c.head_dim, c.n_kv_heads * c.head_dim
        self.fused = fused and c.hidden <= 4096
        self.x = torch.zeros(c.hidden, **f32)             # residual stream
        self.x2 = torch.zeros(c.hidden, **f32)            # its other buffer (fused norms)
        self.rope_epi = rope_rows_interleaved
        assert not self.rope_epi or self.fused, "the RoPE epilogue runs in the fused q/k/v GEMV"
        assert not (self.rope_epi and any(ly.q_norm is not None for ly in layers)), \
            "per-head q/k norms need whole heads: use the RoPE kernel (rows not interleaved)"
        # (cos, sin) of every cache position, built once: read by the q/k/v
        # GEMV's RoPE epilogue and by the prompt path's RoPE kernel.
        # every RoPE of the step and of the prompt path reads this table
        self.rope_tab = (B.qdec_rope_table(max_len, c.head_dim, c.theta, device=dev) if c.rope_scaling is None else
                         B.qdec_rope_table_llama3(max_len, c.head_dim, c.theta, c.rope_scaling, device=dev))
        self.h = torch.zeros(c.hidden, **f16)             # normed input of a projection
        self.q, self.k, self.v = torch.zeros(qd, **f32), torch.zeros(kvd, **f32), torch.zeros(kvd, **f32)
        self.q16 = torch.zeros((c.n_q_heads, c.head_dim), **f16)
        self.attn16 = torch.zeros((c.n_q_heads, c.head_dim), **f16)
        self.y_attn = torch.zeros(c.hidden, **f32)
        self.g16 = torch.zeros(c.inter, **f16)
        self.y_ffn = torch.zeros(c.hidden, **f32)
        self.logits = torch.zeros(c.vocab, **f32)
        self.token = torch.zeros(1, dtype=torch.int32, device=dev)
        self.k_cache = torch.zeros((c.layers, c.n_kv_heads, max_len, c.head_dim), **f16)
        self.v_cache = torch.zeros((c.layers, c.n_kv_heads, max_len, c.head_dim), **f16)
        self.ws = torch.empty(B.qattn_decode_workspace_bytes(c.n_q_heads, c.head_dim), dtype=torch.uint8,
                              device=dev)
        self.argmax_ws = torch.empty(B.ARGMAX_WORKSPACE_BYTES, dtype=torch.uint8, device=dev)
        self.scale = 1.0 / math.sqrt(c.head_dim)

    def step(self, pos: int, stream=None) -> None:
        """Consumes self.token (the token at position pos), writes row pos of
        every layer's caches, self.logits, and the greedy next token into
        self.token."""
        c, s = self.cfg, stream
        B.qdec_embed(self.emb, self.token, out=self.x, stream=s)
        if self.fused:
            for li, ly in enumerate(self.layers):
                res = self.y_ffn if li else None
                if self.rope_epi:
                    # x2 = x + y_ffn; q, k, v = W . norm(x2), rotated, k and v into the caches
                    B.qmatmul_gemv_qkv_rmsnorm_rope([ly.wq, ly.wk, ly.wv], self.x, ly.attn_norm, c.eps, self.x2, pos,
                                                    self.rope_tab, self.q16, self.k_cache[li], self.v_cache[li],
                                                    residual=res, stream=s)
                else:
                    # x2 = x + y_ffn; q, k, v = W . norm(x2)
                    B.qmatmul_gemv_grouped_rmsnorm([ly.wq, ly.wk, ly.wv], self.x, ly.attn_norm, c.eps, self.x2,
                                                   residual=res, outs=[self.q, self.k, self.v], stream=s)
                    # RoPE (with the Qwen3 per-head norms) + cache append, then attention
                    B.qdec_rope_append(self.q, self.k, self.v, pos, c.theta, self.k_cache[li], self.v_cache[li],
                                       q_out=self.q16, q_norm=ly.q_norm, k_norm=ly.k_norm, eps=c.eps,
                                       table=self.rope_tab, stream=s)
                B.qattn_decode(self.q16, self.k_cache[li], self.v_cache[li], pos + 1, self.scale, out=self.attn16,
                               workspace=self.ws, stream=s)
                B.qmatmul_gemv(ly.wo, self.attn16.view(-1), out=self.y_attn, stream=s)
                # x = x2 + y_attn; g = swiglu(norm(x))
                B.qmatmul_gemv_swiglu_rmsnorm_f16(ly.wg, ly.wu, self.x2, ly.ffn_norm, c.eps, self.x,
                                                  residual=self.y_attn, out=self.g16, stream=s)
                B.qmatmul_gemv(ly.wd, self.g16, out=self.y_ffn, stream=s)
            self._head(s)
            return
        for li, ly in enumerate(self.layers):
            B.qdec_rmsnorm(self.x, ly.attn_norm, c.eps, residual=self.y_ffn if li else None, out=self.h, stream=s)
            B.qmatmul_gemv_grouped([ly.wq, ly.wk, ly.wv], [self.h] * 3, [self.q, self.k, self.v], stream=s)
            B.qdec_rope_append(self.q, self.k, self.v, pos, c.theta, self.k_cache[li], self.v_cache[li],
                               q_out=self.q16, q_norm=ly.q_norm, k_norm=ly.k_norm, eps=c.eps,
                               table=self.rope_tab, stream=s)
            B.qattn_decode(self.q16, self.k_cache[li], self.v_cache[li], pos + 1, self.scale, out=self.attn16,
                           workspace=self.ws, stream=s)
            B.qmatmul_gemv(ly.wo, self.attn16.view(-1), out=self.y_attn, stream=s)
            B.qdec_rmsnorm(self.x, ly.ffn_norm, c.eps, residual=self.y_attn, out=self.h, stream=s)
            B.qmatmul_gemv_swiglu(ly.wg, ly.wu, self.h, out=self.g16, stream=s)
            B.qmatmul_gemv(ly.wd, self.g16, out=self.y_ffn, stream=s)
        self._head(s)

    def _head(self, s) -> None:
        B.qdec_rmsnorm(self.x, self.norm, self.cfg.eps, residual=self.y_ffn, out=self.h, stream=s)
        B.qmatmul_gemv(self.lm_head, self.h, out=self.logits, stream=s)
        B.qdec_argmax(self.logits, out=self.token, workspace=self.argmax_ws, stream=s)

    def _chunk_buffers(self, m: int) -> dict:
        """Views of the prompt-chunk buffers for m rows.  The buffers hold
        max_chunk rows and are allocated on the first prefill only (a decoder
        that never prefills pays nothing), so later chunks allocate nothing
        (Sec. 3.2: no allocation in the loop; Sec. 3.4: bounded chunks)."""
        c = self.cfg
        qd, kvd = c.n_q_heads * c.head_dim, c.n_kv_heads * c.head_dim
        shapes = dict(x=((c.hidden,), torch.float32), h=((c.hidden,), torch.float16),
                      q=((qd,), torch.float32), k=((kvd,), torch.float32), v=((kvd,), torch.float32),
                      qh=((qd,), torch.float16), o16=((qd,), torch.float16),
                      ya=((c.hidden,), torch.float32), sw=((c.inter,), torch.float16),
                      y=((c.hidden,), torch.float32))
        if self._chunk is None:
            dev = self.emb.device
            self._chunk = {n: torch.empty(self.max_chunk * sh[0], dtype=dt, device=dev)
                           for n, (sh, dt) in shapes.items()}
            # Key-split partials of the prefill attention, sized for a full
            # chunk at position 0 (the deepest causal triangle); other chunks
            # split within it.
            nb = B.qattn_prefill_workspace_bytes(c.n_q_heads, c.head_dim, self.max_chunk, 0)
            self._chunk["attn_ws"] = torch.empty(max(nb, 16), dtype=torch.uint8, device=dev)
        b = self._chunk
        rows = lambda n: b[n][:m * shapes[n][0][0]].view(m, shapes[n][0][0])
        heads = lambda n: b[n][:m * qd].view(c.n_q_heads, m, c.head_dim)
        out = {n: rows(n) for n in shapes if n != "qh"}
        out.update(qh=heads("qh"), attn_ws=b["attn_ws"])
        return out

    def prefill(self, tokens: torch.Tensor, p0: int = 0, stream=None) -> None:
        """A prompt chunk (Sec. 3.4): tokens (int32 [m], device, 1 <= m <=
        max_chunk) at positions p0 .. p0 + m - 1 through every layer with the
        prefill GEMMs and causal attention; writes those cache rows, the last
        token's logits and the greedy next token into self.token.  Longer
        prompts go through in several chunks."""
        c, s = self.cfg, stream
        m = tokens.numel()
        if not 1 <= m <= self.max_chunk:
            raise ValueError(f"prefill chunk of {m} tokens: must be 1 .. max_chunk={self.max_chunk}")
        b = self._chunk_buffers(m)
        x = B.qdec_embed_rows(self.emb, tokens, out=b["x"], stream=s)     # fp32 [m][H] residual stream
        y = None
        for li, ly in enumerate(self.layers):
            h = B.qdec_rmsnorm(x, ly.attn_norm, c.eps, residual=y, out=b["h"], stream=s)
            q, k, v = B.qmatmul_gemm_grouped([ly.wq, ly.wk, ly.wv], h, outs=[b["q"], b["k"], b["v"]], stream=s)
            qh = B.qdec_rope_append_rows(q, k, v, p0, c.theta, self.k_cache[li], self.v_cache[li],
                                         interleaved=self.rope_epi, q_out=b["qh"], q_norm=ly.q_norm,
                                         k_norm=ly.k_norm, eps=c.eps, table=self.rope_tab, stream=s)
            o16 = B.qattn_prefill_rows_f16(qh, self.k_cache[li], self.v_cache[li], p0, self.scale, out=b["o16"],
                                           workspace=b["attn_ws"], stream=s)
            ya = B.qmatmul_gemm(ly.wo, o16, out=b["ya"], stream=s)
            h = B.qdec_rmsnorm(x, ly.ffn_norm, c.eps, residual=ya, out=b["h"], stream=s)
            sw = B.qmatmul_gemm_swiglu_f16(ly.wg, ly.wu, h, out=b["sw"], stream=s)
            y = B.qmatmul_gemm(ly.wd, sw, out=b["y"], stream=s)
        B.qdec_rmsnorm(x[m - 1], self.norm, c.eps, residual=y[m - 1], out=self.h, stream=s)
        B.qmatmul_gemv(self.lm_head, self.h, out=self.logits, stream=s)
        B.qdec_argmax(self.logits, out=self.token, workspace=self.argmax_ws, stream=s)


class BatchDecoder:
    """Many requests decoded together over a paged KV cache: one step takes
    any number of new tokens of every request (a prompt, a chunk of one, the
    next token), through the prefill GEMMs, qkv_rope_append and
    qattn_paged_f16, and leaves every request's next token.

    Weights as for DenseDecoder.  n_req: requests at most (slots); n_pages:
    pages of page_size tokens that they share; max_len: tokens of one request
    at most (rounded up to pages); max_tokens: new tokens of one step at most,
    all requests together (32,768 or fewer are run).  Which request holds which pages, lengths and
    positions live on the device (qkv_plan), and a step leaves them where it
    found them, so a step (or several) can be captured in a HIP graph and
    replayed between eager steps in any order.  plan: the last step's lengths,
    refusals, offsets and free ring, replayed or not; its positions and slots
    are as many as the last call of step had tokens."""

    def __init__(self, cfg: DecoderConfig, emb: torch.Tensor, layers: List[LayerWeights], norm: torch.Tensor,
                 lm_head: B.QWeight, n_req: int, n_pages: int, max_len: int, page_size: int = 64,
                 max_tokens: int = 2048, rope_rows_interleaved: bool = False):
        if rope_rows_interleaved and any(ly.q_norm is not None for ly in layers):
            raise ValueError("per-head q/k norms need rows that are not interleaved")
        self.cfg, self.emb, self.layers, self.norm, self.lm_head = cfg, emb, layers, norm, lm_head
        self.n_req, self.page_size, self.max_tokens = n_req, page_size, max_tokens
        self.interleaved = rope_rows_interleaved
        max_pages = -(-max_len // page_size)
        dev, c = emb.device, cfg
        f32, f16, i32 = (dict(dtype=t, device=dev) for t in (torch.float32, torch.float16, torch.int32))
        qd, kvd = c.n_q_heads * c.head_dim, c.n_kv_heads * c.head_dim
        table_len = max_pages * page_size
        self.rope_tab = (B.qdec_rope_table(table_len, c.head_dim, c.theta, device=dev) if c.rope_scaling is None else
                         B.qdec_rope_table_llama3(table_len, c.head_dim, c.theta, c.rope_scaling, device=dev))
        pool = (c.layers, n_pages, c.n_kv_heads, page_size, c.head_dim)
        self.k_pages, self.v_pages = torch.zeros(pool, **f16), torch.zeros(pool, **f16)
        self.tables = torch.full((n_req, max_pages), -1, **i32)
        self.free_ring = torch.arange(n_pages, **i32)            # every page is free
        self.prefix: Optional[torch.Tensor] = None               # page ids that all requests share
        self._captured = False                                   # a graph holds a step (with this prefix)
        # Lengths, and the free ring's head and count, before a step and behind it: qkv_plan writes other
        # places than it reads, and the step brings its result back to where the next one looks.
        self._before, self._behind = (torch.zeros(n_req + 2, **i32) for _ in range(2))
        self._before[-1] = n_pages
        self._behind[-1] = n_pages
        plan = B.empty_kv_plan(n_req, 0, device=dev)
        self.plan = replace(plan, lens=self._behind[:n_req], ring=self._behind[n_req:])   # the last step's
        self._positions = torch.empty(max_tokens, **i32)
        self._slots = torch.empty(max_tokens, dtype=torch.int64, device=dev)
        self.x = torch.zeros((max_tokens, c.hidden), **f32)      # residual stream
        # Normed input of a projection, behind a row of zeros: row offsets[i + 1] is request i's last token.
        self.h = torch.zeros((1 + max_tokens, c.hidden), **f16)
        self.q, self.k, self.v = (torch.zeros((max_tokens, n), **f32) for n in (qd, kvd, kvd))
        self.q16 = torch.zeros((max_tokens, c.n_q_heads, c.head_dim), **f16)
        self.o16 = torch.zeros((max_tokens, qd), **f16)
        self.y_attn, self.y_ffn = (torch.zeros((max_tokens, c.hidden), **f32) for _ in range(2))
        self.g16 = torch.zeros((max_tokens, c.inter), **f16)
        self.last = torch.zeros((n_req, c.hidden), **f32)
        # Normed last token: of the rows of this step, and of every request's last step with tokens.
        self.step16, self.last16 = (torch.zeros((n_req, c.hidden), **f16) for _ in range(2))
        self.logits = torch.zeros((n_req, c.vocab), **f32)
        self.token = torch.zeros(n_req, **i32)                   # greedy next token of every request
        self.ws = torch.empty(B.qattn_paged_workspace_bytes(c.n_q_heads, c.n_kv_heads, c.head_dim, n_req, max_tokens, 1),
                              dtype=torch.uint8, device=dev)
        self.ws_plain = torch.empty(B.qattn_paged_workspace_bytes(c.n_q_heads, c.n_kv_heads, c.head_dim, n_req,
                                                                  max_tokens), dtype=torch.uint8, device=dev)
        self.argmax_ws = torch.empty(B.qdec_argmax_rows_workspace_bytes(n_req), dtype=torch.uint8, device=dev)
        self.scale = 1.0 / math.sqrt(c.head_dim)

    def step(self, tokens: torch.Tensor, new_lens: torch.Tensor, stream=None) -> None:
        """tokens: int32 [T] on the device, T <= max_tokens, the requests' new
        tokens one after the other in the order of the slots (places behind
        the last one count nothing); new_lens: int32 [n_req], how many each
        request has (0: none; -1: it has ended, its pages are free from the
        next step on).  Leaves logits and the greedy next token of every
        request with new tokens in self.logits[i] and self.token[i]; the others
        keep theirs.  A request that finds no pages is refused
        (self.plan.refused, kv_lens 0): its tokens are not cached, and it keeps
        its logits and next token too, so the same tokens can come again."""
        c, s, t = self.cfg, stream, tokens.numel()
        if not 1 <= t <= self.max_tokens:
            raise ValueError(f"a step of {t} tokens: must be 1 .. max_tokens={self.max_tokens}")
        if tokens.dtype != torch.int32 or tokens.device != self.emb.device or not tokens.is_contiguous():
            raise ValueError(f"tokens: need contiguous int32 on {self.emb.device}, got {tokens.dtype} on {tokens.device}")
        x, h, y = self.x[:t], self.h[1:1 + t], None
        ws = self.ws_plain if self.prefix is None else self.ws
        B.qdec_embed_rows(self.emb, tokens, out=x, stream=s)
        plan = replace(self.plan, positions=self._positions[:t], slots=self._slots[:t])
        n = self.n_req
        B.qkv_plan(self._before[:n], new_lens, self.tables, self.free_ring, self._before[n:], self.page_size, t,
                   prefix_pages=0 if self.prefix is None else self.prefix.numel(), out=plan, stream=s)
        self.plan = plan                                         # (a refused call leaves everything as it was)
        with torch.cuda.stream(s):
            self._before.copy_(self._behind)
            self._captured = self._captured or torch.cuda.is_current_stream_capturing()
        for li, ly in enumerate(self.layers):
            B.qdec_rmsnorm(x, ly.attn_norm, c.eps, residual=y, out=h, stream=s)
            q, k, v = B.qmatmul_gemm_grouped([ly.wq, ly.wk, ly.wv], h, outs=[self.q[:t], self.k[:t], self.v[:t]],
                                             stream=s)
            B.qkv_rope_append(q, k, v, plan.positions, plan.slots, self.rope_tab, self.k_pages[li], self.v_pages[li],
                              interleaved=self.interleaved, q_norm=ly.q_norm, k_norm=ly.k_norm, eps=c.eps,
                              q_out=self.q16[:t], stream=s)
            B.qattn_paged_f16(self.q16[:t], self.k_pages[li], self.v_pages[li], self.tables, plan.offsets,
                              plan.kv_lens, self.scale, prefix=self.prefix, out=self.o16[:t], workspace=ws, stream=s)
            B.qmatmul_gemm(ly.wo, self.o16[:t], out=self.y_attn[:t], stream=s)
            B.qdec_rmsnorm(x, ly.ffn_norm, c.eps, residual=self.y_attn[:t], out=h, stream=s)
            B.qmatmul_gemm_swiglu_f16(ly.wg, ly.wu, h, out=self.g16[:t], stream=s)
            y = B.qmatmul_gemm(ly.wd, self.g16[:t], out=self.y_ffn[:t], stream=s)
        B.qdec_rmsnorm(x, self.norm, c.eps, residual=y, out=h, stream=s)
        B.qdec_embed_rows(self.h[:1 + t], plan.offsets[1:], out=self.last, stream=s)
        B.qdec_cast_f16(self.last, out=self.step16, stream=s)
        with torch.cuda.stream(s):
            served = torch.minimum(new_lens, plan.kv_lens) > 0   # new tokens, and not refused
            torch.where(served[:, None], self.step16, self.last16, out=self.last16)
        B.qmatmul_gemm(self.lm_head, self.last16, out=self.logits, stream=s)
        B.qdec_argmax_rows(self.logits, out=self.token, workspace=self.argmax_ws, stream=s)

    def share_prefix(self, tokens: torch.Tensor, stream=None) -> None:
        """Before any other step (or capture of one): runs tokens (int32 [n] on
        the device, n a multiple of page_size) once and keeps them as the
        beginning of every request.  Waits for the device."""
        n, pages = tokens.numel(), tokens.numel() // self.page_size
        if self.prefix is not None or n == 0 or n % self.page_size or n > self.tables.shape[1] * self.page_size:
            raise ValueError(f"a prefix of {n} tokens: one, of whole pages of {self.page_size}, within max_len")
        if self._captured:
            raise ValueError("a prefix comes before a step is captured: the graph goes on without it")
        with torch.cuda.stream(stream):
            if self.plan.lens.any().item() or self.plan.ring[1].item() < pages:
                raise ValueError(f"a prefix comes before any other step and has to find its {pages} pages")
            for at in range(0, n, self.max_tokens):
                part = tokens[at:at + self.max_tokens]
                new = torch.zeros(self.n_req, dtype=torch.int32, device=tokens.device)
                new[0] = part.numel()
                self.step(part, new, stream=stream)
            self.prefix = self.tables[0, :pages].clone()
            self.tables[:, :pages] = self.prefix
            torch.cuda.current_stream().synchronize()
