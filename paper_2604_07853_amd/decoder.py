"""A decoder layer on the library's own kernels: what a rollout engine (a few tokens per call) and the learner's forward (whole prompts) run.

    residual add + RMS norm -> q, k, v projection -> paged cache (written quantized or plain) -> attention over it -> o projection
    -> residual add + RMS norm (its output also as the experts' e4m3 rows) -> router -> quantized experts

The projections are the grouped GEMM with one expert, on bf16 rows: W4A16 weights.  Positions are the caller's: `rotate(q, k)`, called on the views of the
new tokens' queries and keys before they are cached, applies what the model uses.  The router's logits are a plain library product.
"""
import torch

from . import binding as q


class DecoderLayer:
    """norm1, norm2 bf16 [H]; qkv QWeight [1, (heads + 2 kv_heads) * head_dim, H]; o QWeight [1, H, heads * head_dim], both W4A16; router bf16
    [experts, H]; gate_up, down the experts' QWeights, of any format; cache a KVCache of this layer."""

    def __init__(self, norm1, qkv, o, norm2, router, gate_up, down, cache, topk=8, eps=1e-6):
        D = cache.head_dim
        self.H, self.heads = o.N, o.K // D
        if (qkv.E, qkv.N, qkv.K) != (1, (self.heads + 2 * cache.kv_heads) * D, self.H) or o.E != 1 or o.K != self.heads * D:
            raise ValueError("qkv and o must be one matrix each, [(heads + 2 kv_heads) * head_dim, H] and [H, heads * head_dim] (got %s, %s)"
                             % ((qkv.E, qkv.N, qkv.K), (o.E, o.N, o.K)))
        if qkv.fmt in q.E4M3_ACT_FORMATS or o.fmt in q.E4M3_ACT_FORMATS:
            raise ValueError("qkv and o run on bf16 rows: QARL_W4A16_G128 weights (got formats %d, %d)" % (qkv.fmt, o.fmt))
        if self.heads % cache.kv_heads:
            raise ValueError("%d query heads on %d cached ones" % (self.heads, cache.kv_heads))
        if norm1.shape != (self.H,) or norm2.shape != (self.H,) or router.shape != (gate_up.E, self.H) or gate_up.K != self.H:
            raise ValueError("norms must be [%d], router [%d, %d] and gate_up of K = %d" % (self.H, gate_up.E, self.H, self.H))
        # the experts' kernels write down's rows and columns into the layer's own buffers
        if (down.E, down.N, 2 * down.K) != (gate_up.E, self.H, gate_up.N) or (gate_up.fmt in q.E4M3_ACT_FORMATS) != (down.fmt in q.E4M3_ACT_FORMATS):
            raise ValueError("down must be [%d, %d, %d] on rows of gate_up's kind (got %s, formats %d and %d)"
                             % (gate_up.E, self.H, gate_up.N // 2, (down.E, down.N, down.K), gate_up.fmt, down.fmt))
        if gate_up.E % 64 or gate_up.E > 256 or not 1 <= topk <= min(gate_up.E, 32):
            raise ValueError("the router takes 64, 128, 192 or 256 experts and picks 1 to 32 (got %d, %d)" % (gate_up.E, topk))
        self.norm1, self.qkv, self.o, self.norm2, self.router = norm1, qkv, o, norm2, router
        self.gu, self.dn, self.cache, self.topk, self.eps = gate_up, down, cache, topk, eps
        self.e4m3_rows = gate_up.fmt in q.E4M3_ACT_FORMATS
        self._moe = {}          # decode batches, up to 512 tokens: the experts' layer object by number of tokens,
        self._room = None       # all on the buffers of the largest (a server meets every number of them, and a captured step keeps its addresses)
        self._stream = None     # the stream that last used those buffers, and its handle
        self._handle = None
        self._one = {}          # and the row offsets of a projection, [0, T]

    def _project(self, W, x):
        T = x.shape[0]
        offsets = self._one.get(T)
        if offsets is None:
            offsets = torch.arange(2, dtype=torch.int32, device=x.device).mul_(T)       # made on the GPU: a graph capture takes no copy from the host
            if T <= 512 and not torch.cuda.is_current_stream_capturing():               # (and fills what it makes when it is replayed)
                self._one[T] = offsets
        return q.qarl_qgemm_grouped(W, x, offsets, T)

    def _take_buffers(self, y):
        """The buffers of batches of up to 512 belong to one call at a time: a call on another stream waits for what the last one's stream holds."""
        handle = torch._C._cuda_getCurrentRawStream(y.get_device())
        if handle == self._handle or torch.cuda.is_current_stream_capturing():      # (a graph's replays are ordered by whoever replays it)
            return
        stream = torch.cuda.current_stream(y.device)
        if self._stream is not None:
            stream.wait_stream(self._stream)
        self._stream, self._handle = stream, handle

    def _experts(self, y, codes, scales):
        T = y.shape[0]
        logits = torch.matmul(y, self.router.t())
        if T <= 512:
            self._take_buffers(y)
        if codes is None:
            moe = self._moe.get(T)
            if moe is None:     # few tokens: one call, the experts' kernels read (and quantize) the bf16 rows themselves
                moe = q.MoELayer(self.gu, self.dn, T, self.topk, q.QARL_PATH_DECODE if T <= 512 else q.QARL_PATH_PREFILL, y.device)
                if T <= 512:
                    if self._room is None:
                        self._room = q.MoELayer(self.gu, self.dn, 512, self.topk, q.QARL_PATH_DECODE, y.device)
                    moe.a, moe.out = self._room.a[: moe.M], self._room.out[:T]
                    if moe.ws.numel() <= self._room.ws.numel():
                        moe.ws = self._room.ws
                    self._moe[T] = moe
            return moe.forward(y, logits)
        r = q.qarl_moe_route(logits, self.topk)
        M = T * self.topk
        a = q.qarl_qgemm_grouped(self.gu, codes, r.offsets, M, row_map=r.tokens, x_scales=scales, epilogue=q.QARL_EPI_SILU_MUL, path=q.QARL_PATH_PREFILL)
        aq, sa = q.qarl_quantize_rows_fp8(a)
        return q.qarl_qgemm_grouped(self.dn, aq, r.offsets, M, x_scales=sa, epilogue=q.QARL_EPI_COMBINE, combine_w=r.w, sorted_pairs=r.pairs, T=T,
                                    topk=self.topk, path=q.QARL_PATH_PREFILL)

    def forward(self, x, residual, slots, block_table, kv_lens, q_offsets, max_q_len, max_kv_len, window=0, rotate=None):
        """x [T, H] bf16: what the layer before has computed; residual [T, H]: the residual stream so far (None in front of the first layer).  slots,
        block_table, kv_lens, q_offsets, max_q_len, max_kv_len: as for qarl_kv_cache_write and qarl_paged_attention, kv_lens with the new tokens.
        Returns (output, residual) for the next layer, whose first norm adds them.  Up to 512 tokens the output is the layer's own buffer, written
        again by its next call of up to 512, on whatever stream: such calls wait for the stream of the call before (and for its reader there); the replays
        of a captured step and other calls are for the caller to order."""
        T, c = x.shape[0], self.cache
        n1 = q.qarl_add_rmsnorm(x, self.norm1, self.eps, residual=residual)
        residual = x if residual is None else n1["residual"]
        heads = self._project(self.qkv, n1["y"]).view(T, self.heads + 2 * c.kv_heads, c.head_dim)
        query, key, value = heads.split([self.heads, c.kv_heads, c.kv_heads], 1)
        if rotate is not None:
            query, key = rotate(query, key)
        q.qarl_kv_cache_write(c, key, value, slots)
        att = q.qarl_paged_attention(query, c, block_table, kv_lens, q_offsets, max_q_len, max_kv_len, window=window)["out"]
        out = self._project(self.o, att.view(T, self.heads * c.head_dim))
        # whole prompts on e4m3 rows: the norm quantizes them on the way, to the bytes that the decode path makes of its bf16 rows
        fused = self.e4m3_rows and T > 512
        y = torch.empty_like(out)
        n2 = q.qarl_add_rmsnorm(out, self.norm2, self.eps, residual=residual, y=y, quantize=fused, via_bf16=True)
        return self._experts(y, n2["codes"], n2["scales"]), n2["residual"]
