"""Device-memory plumbing around the binding: moves a generated workload to the
GPU, allocates outputs and workspace with torch, and issues the library calls.
No arithmetic of the method happens here."""
from __future__ import annotations

import dataclasses
from typing import Optional

import numpy as np
import torch

from . import binding as B


def _dev(a: Optional[np.ndarray], device, bf16: bool = False):
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a))
    if bf16:
        t = t.view(torch.int16).view(torch.bfloat16)
    return t.to(device)


@dataclasses.dataclass
class DeviceAttn:
    desc: B.AttnDesc
    q: torch.Tensor
    k_prefix: torch.Tensor
    v_prefix: torch.Tensor
    prefix_lens: torch.Tensor
    prefix_indptr: torch.Tensor
    prefix_page_indices: Optional[torch.Tensor]
    sample_indptr: torch.Tensor
    k_suffix: torch.Tensor
    v_suffix: torch.Tensor
    suffix_lens: torch.Tensor
    suffix_page_indptr: Optional[torch.Tensor]
    suffix_page_indices: Optional[torch.Tensor]
    max_prefix_len: int
    max_suffix_len: int
    out: torch.Tensor
    lse: torch.Tensor
    workspace: torch.Tensor

    def run(self, stages: int = 0, stream=None) -> None:
        self.desc.stages = stages
        B.shared_prefix_decode_attn(
            self.desc, self.q, self.k_prefix, self.v_prefix, self.prefix_lens, self.prefix_indptr,
            self.prefix_page_indices, self.sample_indptr, self.k_suffix, self.v_suffix,
            self.suffix_lens, self.suffix_page_indptr, self.suffix_page_indices,
            self.max_prefix_len, self.max_suffix_len, self.out, self.lse, self.workspace, stream)


def upload_attn(inp, device="cuda:0", workspace: Optional[torch.Tensor] = None) -> DeviceAttn:
    """Copy an AttnInputs record to the GPU and allocate output + workspace."""
    sp = inp.spec
    bf16 = sp.dtype == "bf16"
    paged = sp.page_size != 0
    desc = B.make_desc(dtype=B.SPD_BF16 if bf16 else B.SPD_F32, num_q_heads=sp.num_q_heads,
                       num_kv_heads=sp.num_kv_heads, head_dim=sp.head_dim,
                       num_prompts=sp.num_prompts, num_samples=sp.num_samples,
                       max_samples_per_prompt=sp.samples_per_prompt, page_size=sp.page_size)
    kp, vp = _dev(inp.k_prefix, device, bf16), _dev(inp.v_prefix, device, bf16)
    if paged and inp.k_suffix is inp.k_prefix:
        ks, vs = kp, vp
    else:
        ks, vs = _dev(inp.k_suffix, device, bf16), _dev(inp.v_suffix, device, bf16)
    N, Hq, D = inp.q.shape
    out = torch.empty((N, Hq, D), dtype=torch.bfloat16 if bf16 else torch.float32, device=device)
    lse = torch.empty((N, Hq), dtype=torch.float32, device=device)
    if workspace is None:
        nbytes = B.shared_prefix_decode_attn_workspace_size(desc, inp.max_prefix_len, inp.max_suffix_len)
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return DeviceAttn(desc, _dev(inp.q, device, bf16), kp, vp, _dev(inp.prefix_lens, device),
                      _dev(inp.prefix_indptr, device), _dev(inp.prefix_page_indices, device),
                      _dev(inp.sample_indptr, device), ks, vs, _dev(inp.suffix_lens, device),
                      _dev(inp.suffix_page_indptr, device), _dev(inp.suffix_page_indices, device),
                      inp.max_prefix_len, inp.max_suffix_len, out, lse, workspace)


@dataclasses.dataclass
class DeviceSampler:
    logits: torch.Tensor
    temperature: torch.Tensor
    top_p: torch.Tensor
    uniforms: torch.Tensor
    tokens: torch.Tensor
    workspace: torch.Tensor

    def run(self, stream=None) -> None:
        rows, vocab = self.logits.shape
        B.sample_tokens(self.logits, B.SPD_F32, rows, vocab, self.logits.stride(0), self.temperature,
                        self.top_p, self.uniforms, self.tokens, self.workspace, stream)


def upload_sampler(inp, device="cuda:0", row_stride=None, pad_value=float("nan")) -> DeviceSampler:
    """Uploads sampler inputs.  With `row_stride` > vocab the logits sit in a wider matrix whose
    extra columns hold `pad_value` (the kernels must never read them as logits)."""
    rows, vocab = inp.logits.shape
    ws = torch.empty(max(256, B.sample_tokens_workspace_size(rows, vocab)), dtype=torch.uint8, device=device)
    if row_stride is not None and row_stride != vocab:
        wide = torch.full((rows, row_stride), pad_value, dtype=torch.float32, device=device)
        wide[:, :vocab] = _dev(inp.logits, device)
        logits = wide[:, :vocab]  # a view: stride(0) == row_stride
    else:
        logits = _dev(inp.logits, device)
    return DeviceSampler(logits, _dev(inp.temperature, device), _dev(inp.top_p, device),
                         _dev(inp.uniforms, device), torch.empty(rows, dtype=torch.int32, device=device), ws)


def _require(ok: bool, message: str) -> None:
    if not ok:
        raise ValueError(message)


def _on_one_gpu(*tensors) -> bool:
    return all(t.is_cuda and t.device == tensors[0].device for t in tensors if t is not None)


def _torch_stream(stream, device):
    """`stream` as the allocator knows it: None, a torch stream, or one made elsewhere (an object with its handle, or that)."""
    if stream is None or isinstance(stream, torch.cuda.Stream):
        return stream
    handle = B._stream(stream)
    return torch.cuda.ExternalStream(handle, device) if handle else torch.cuda.default_stream(device)


@dataclasses.dataclass
class PageTables:
    """What `build_page_tables` leaves for a batch of requests (all on the device)."""
    page_indptr: torch.Tensor
    page_indices: torch.Tensor
    lens: torch.Tensor        # tokens each request may hold now
    new_indptr: torch.Tensor  # running count of new tokens granted
    slots: Optional[torch.Tensor]  # of the rows that packed_indptr counts
    free_end: torch.Tensor    # first page of the free list not dealt
    page_size: int = 16
    packed_indptr: Optional[torch.Tensor] = None  # running count of new tokens asked for: rows are packed by it
    packed_lens: Optional[torch.Tensor] = None    # `lens`, 0 for refused requests


def build_tables(lens, free_pages, max_pages: int, max_tokens: int = 0, page_size: int = 16, held: Optional[PageTables] = None,
                 free_begin=None, stream=None) -> PageTables:
    """Page tables of requests that have to hold `lens` tokens (device int32), dealt from `free_pages`.  `held`: the
    tables the same requests have so far; `free_begin`: another call's `free_end`.  max_tokens 0: no slot map and no packed_*.
    The rows of new tokens (q, k, v, ids) are packed by what `lens` asks for beyond `held`, granted or not.
    The tables and the workspace are allocated here, on `stream` where one is given, so that their memory is not handed
    out again before it is done with them (nor, when the tables go, before what the current stream then holds)."""
    ints = {"lens": (lens, 1), "free_pages": (free_pages, 0), "free_begin": (free_begin, 1)}
    if held is not None:
        _require(held.page_size == page_size and held.lens.numel() == lens.numel(), "held tables are of the same requests and page size")
        ints.update({"held lens": (held.lens, 1), "held page_indptr": (held.page_indptr, lens.numel() + 1),
                     "held page_indices": (held.page_indices, 0)})
    for name, (x, least) in ints.items():
        _require(x is None or (x.dtype == torch.int32 and x.is_contiguous() and x.numel() >= least),
                 f"{name} has to be contiguous int32 of {least} or more")
    _require(_on_one_gpu(*(x for x, _ in ints.values())), "everything has to be on one GPU")
    n, dev = lens.numel(), lens.device
    empty = lambda k, t=torch.int32: torch.empty(k, dtype=t, device=dev)
    with torch.cuda.stream(_torch_stream(stream, dev)):  # (nothing where it is None)
        out = PageTables(empty(n + 1), empty(max_pages), empty(n), empty(n + 1), empty(max_tokens, torch.int64) if max_tokens else None,
                         empty(1), page_size, *((empty(n + 1), empty(n)) if max_tokens else ()))
        ws = empty(B.build_page_tables_workspace_size(n), torch.uint8)
    if stream is not None:
        for x in (out.page_indptr, out.page_indices, out.lens, out.new_indptr, out.slots, out.free_end, out.packed_indptr, out.packed_lens):
            if x is not None and x.numel():
                x.record_stream(torch.cuda.current_stream(dev))
    # (a list without pages has no address; where nobody holds a page, none is read)
    held_pages = held and (held.page_indices if held.page_indices.numel() else held.page_indptr)
    args = (n, page_size, lens, held and held.lens, held and held.page_indptr, held_pages, free_pages,
            free_pages.numel(), free_begin, max_pages, max_tokens, out.page_indptr, out.page_indices, out.lens, out.new_indptr, out.slots,
            out.free_end)
    if max_tokens:
        B.build_page_tables_packed(*args, out.packed_indptr, out.packed_lens, ws, stream)
    else:
        B.build_page_tables(*args, ws, stream)
    return out


class DevicePrompts:
    """One layer's prompt pass on the GPU: stores the new tokens' keys and values in the pages that `tables` name, then
    the attention of the new tokens over everything their prompts hold.  q, k, v: [tokens, heads, head_dim], rows of a
    projection (their token stride may be larger than their heads, k's and v's alike); k_pool, v_pool:
    [pages, kv_heads, 16, head_dim].  The rows are packed as the tables were asked for: a refused request's keep their places,
    are stored nowhere, and get zeros (and -inf).  What the kernels could not read as it lies raises ValueError."""

    def __init__(self, tables: PageTables, q, k, v, k_pool, v_pool, max_query_len: int, max_kv_len: int, causal: bool = True,
                 sm_scale: float = 0.0):
        self._check(tables, q, k, v, k_pool, v_pool)
        tokens, hq, d = q.shape
        hkv = k.shape[1]
        self.tables, self.q, self.k, self.v, self.k_pool, self.v_pool = tables, q, k, v, k_pool, v_pool
        self.max_query_len, self.max_kv_len = max_query_len, max_kv_len
        self.desc = B.make_prompt_desc(dtype=B.SPD_BF16 if q.dtype == torch.bfloat16 else B.SPD_F32, num_q_heads=hq, num_kv_heads=hkv,
                                       head_dim=d, num_prompts=tables.lens.numel(), page_size=16, causal=causal, sm_scale=sm_scale,
                                       q_stride=q.stride(0) if tokens > 1 else 0, kv_stride=k.stride(0) if tokens > 1 else 0)
        self.out = torch.empty((tokens, hq, d), dtype=q.dtype, device=q.device)
        self.lse = torch.empty((tokens, hq), dtype=torch.float32, device=q.device)
        size = B.prompt_attn_workspace_size(self.desc, tokens, max_query_len, max_kv_len)
        self.workspace = torch.empty(max(size, 256), dtype=torch.uint8, device=q.device)

    @staticmethod
    def _check(tables: PageTables, q, k, v, k_pool, v_pool) -> None:
        _require(q.dtype in (torch.bfloat16, torch.float32), "q has to be bfloat16 or float32")
        _require(all(x.dtype == q.dtype for x in (k, v, k_pool, v_pool)), "k, v and the pools have to be of q's type")
        _require(q.dim() == 3 and k.dim() == 3 and v.shape == k.shape and k.shape[0] == q.shape[0] and k.shape[2] == q.shape[2],
                 "q is [tokens, heads, head_dim], k and v [tokens, kv_heads, head_dim]")
        tokens, hkv, d = k.shape
        for name, x in (("q", q), ("k", k), ("v", v)):
            _require(x[:1].is_contiguous(), f"{name}'s heads have to follow one another within a token")
            _require(tokens < 2 or x.stride(0) >= x.shape[1] * d, f"{name}'s tokens must not overlap")
        _require(tokens < 2 or k.stride(0) == v.stride(0), "k and v have to have one token stride")
        for x in (k_pool, v_pool):
            _require(x.dim() == 4 and x.shape[1:] == (hkv, 16, d) and x.shape[0] == k_pool.shape[0] and x.is_contiguous(),
                     "the pools are [pages, kv_heads, 16, head_dim], contiguous")
        n = tables.lens.numel()
        _require(tables.page_size == 16, "the tables' pages have to be of 16 tokens")
        _require(tokens == 0 or tables.slots is not None and tables.slots.numel() >= tokens, "the tables need a slot for every token")
        lists = {"lens": n, "new_indptr": n + 1, "page_indptr": n + 1, "page_indices": 0}
        if tables.packed_indptr is not None or tables.packed_lens is not None:
            _require(tables.packed_indptr is not None and tables.packed_lens is not None, "packed_indptr and packed_lens go together")
            lists.update(packed_indptr=n + 1, packed_lens=n)
        _require(all(getattr(tables, x).dtype == torch.int32 and getattr(tables, x).is_contiguous() and getattr(tables, x).numel() >= least
                     for x, least in lists.items()) and
                 (tables.slots is None or tables.slots.dtype == torch.int64 and tables.slots.is_contiguous()),
                 "the tables are int32, the slots int64, contiguous, with an entry for every request")
        _require(_on_one_gpu(q, k, v, k_pool, v_pool, tables.slots, *(getattr(tables, x) for x in lists)),
                 "everything has to be on one GPU")

    def run(self, stream=None) -> None:
        t, tokens = self.tables, self.q.shape[0]
        if tokens == 0:
            return  # (tensors without elements have no address to hand on)
        B.write_prompt_kv(self.desc, self.k, self.v, t.slots, tokens, self.k_pool.shape[0], self.k_pool, self.v_pool, stream)
        starts, lens = (t.new_indptr, t.lens) if t.packed_indptr is None else (t.packed_indptr, t.packed_lens)
        B.prompt_attn(self.desc, self.q, self.k_pool, self.v_pool, starts, lens, t.page_indptr, t.page_indices, tokens,
                      self.max_query_len, self.max_kv_len, self.out, self.lse, self.workspace, stream)


def _check_penalties(sampler: DeviceSampler, raw, penalties: dict) -> None:
    """That `penalize_logits` reads and writes what it is given: types, shapes and strides."""
    to = sampler.logits
    _require(raw.dtype in (torch.bfloat16, torch.float32), "raw_logits have to be bfloat16 or float32")
    _require(to.dtype == torch.float32 and raw.dim() == 2 and raw.shape == to.shape,
             "raw_logits need the shape of the sampler's float32 logits")
    rows, vocab = raw.shape
    _require(sampler.tokens.dtype == torch.int32 and sampler.tokens.is_contiguous() and sampler.tokens.numel() == rows,
             "the sampler needs an int32 token for every row")
    _require(all(x[:1].is_contiguous() and (rows < 2 or x.stride(0) >= vocab) for x in (raw, to)), "a row of logits has to be contiguous")
    (raw_first, raw_end), (to_first, to_end) = ((x.data_ptr(), x.data_ptr() + ((rows - 1) * x.stride(0) + vocab) * x.element_size())
                                                for x in (raw, to))
    _require(raw_first >= to_end or to_first >= raw_end,
             "raw_logits must not share memory with the sampler's: every step shapes them anew")
    words = -(-vocab // 32)
    # type, entries at least
    lists = {"repetition": (torch.float32, rows), "frequency": (torch.float32, rows), "presence": (torch.float32, rows),
             "prompt_of_row": (torch.int32, rows), "allowed_of_row": (torch.int32, rows), "bias_indptr": (torch.int32, rows + 1),
             "bias_tokens": (torch.int32, 0), "bias_values": (torch.float32, 0)}
    for name, x in penalties.items():
        _require(name in lists or name in ("prompt_bits", "allowed_bits"), f"{name} is no penalty that a loop takes")
        if x is None:
            continue
        if name in lists:
            dtype, least = lists[name]
            _require(x.dtype == dtype and x.is_contiguous() and x.numel() >= least,
                     f"{name} has to be contiguous {dtype}, with an entry for every row")
        else:
            least = rows if penalties.get(name.replace("bits", "of_row")) is None else 0
            _require(x.dtype == torch.int32 and x.dim() == 2 and x.shape[1] >= words and x[:1].is_contiguous() and x.shape[0] >= least and
                     (x.shape[0] < 2 or x.stride(0) >= words), f"{name} is int32 [rows, {words} words at least]")
    biases = [penalties.get(x) for x in ("bias_indptr", "bias_tokens", "bias_values")]
    _require(all(x is None for x in biases) or (all(x is not None for x in biases) and biases[1].numel() == biases[2].numel()),
             "bias_indptr, bias_tokens and bias_values go together, a value for every token")
    _require(_on_one_gpu(raw, to, *penalties.values()), "everything has to be on one GPU")


class DeviceLogprobs:
    """How probable given tokens are under their rows' logits, and what stood beside them.  logits: [rows, vocab], fp32 or bf16 (a row
    contiguous); tokens: int32 [rows] on the device, read when `run` is called (a sampler's `tokens`, or a prompt's next ones);
    temperature: float [rows] (a sampler's: 0 counts as 1) or None.  `run` fills logprobs, ranks, entropy, lse [rows] and top_tokens,
    top_logprobs [rows, num_top]."""

    def __init__(self, logits, tokens, temperature=None, num_top: int = 0):
        _require(logits.dtype in (torch.bfloat16, torch.float32) and logits.dim() == 2, "logits are bfloat16 or float32 [rows, vocab]")
        rows, vocab = logits.shape
        _require(logits[:1].is_contiguous() and (rows < 2 or logits.stride(0) >= vocab), "a row of logits has to be contiguous")
        _require(tokens.dtype == torch.int32 and tokens.is_contiguous() and tokens.numel() == rows, "tokens are int32, one for every row")
        _require(temperature is None or temperature.dtype == torch.float32 and temperature.is_contiguous() and temperature.numel() == rows,
                 "temperature is float32, one for every row")
        _require(0 <= num_top <= min(vocab, 64), "num_top is 0 to 64, and no more than the vocabulary")
        _require(_on_one_gpu(logits, tokens, temperature), "everything has to be on one GPU")
        size = B.token_logprobs_workspace_size(rows, vocab, num_top)
        _require(rows == 0 or size > 0, "these are more than token_logprobs takes, or rows of no logits")
        self.logits, self.tokens, self.temperature, self.num_top = logits, tokens, temperature, num_top
        empty = lambda *n, t=torch.float32: torch.empty(n, dtype=t, device=logits.device)  # noqa: E731
        self.logprobs, self.entropy, self.lse = empty(rows), empty(rows), empty(rows)
        self.ranks = empty(rows, t=torch.int32)
        self.top_tokens, self.top_logprobs = empty(rows, num_top, t=torch.int32), empty(rows, num_top)
        self.workspace = empty(max(size, 256), t=torch.uint8)

    def run(self, stream=None) -> None:
        rows, vocab = self.logits.shape
        if rows == 0:
            return  # (tensors without elements have no address to hand on)
        top = (self.top_tokens, self.top_logprobs) if self.num_top else (None, None)
        B.token_logprobs(self.logits, B.SPD_BF16 if self.logits.dtype == torch.bfloat16 else B.SPD_F32, rows, vocab,
                         self.logits.stride(0) if rows > 1 else vocab, self.temperature, self.tokens, self.num_top, self.logprobs,
                         self.ranks, self.entropy, self.lse, *top, self.workspace, stream)


class DeviceEviction:
    """Keeps the private suffixes of a decode call within bounds.  `accumulate`, after the attention of every step, adds what each
    cached token got to its weight (`decay` times what it had); `evict`, when the suffixes are full or before, leaves the `budget` tokens
    of every sample and KV head that weigh most, the first `sinks` and the last `recent` among them, in the front of the sample's own
    slots or pages, and sets suffix_lens.  Weights belong to tokens: they move with them, and a token appended starts from 0.  Where
    suffixes are set back by anything else, `reset` forgets all weights.  The calls launch kernels only and can be captured."""

    def __init__(self, attn: DeviceAttn, budget: int, sinks: int = 4, recent: int = 32, decay: float = 1.0):
        n, hq, d = attn.q.shape
        hkv, room = attn.desc.num_kv_heads, attn.max_suffix_len
        _require(0 < budget <= room, "the budget is 1 to max_suffix_len tokens")
        _require(sinks >= 0 and recent >= 0, "sinks and recent are counts")
        _require(attn.lse is not None, "the decode call has to leave its log-sum-exps")
        dev = attn.q.device
        self.attn, self.budget, self.sinks, self.recent, self.decay = attn, budget, sinks, recent, decay
        self.desc = B.make_prompt_desc(dtype=attn.desc.dtype, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, num_prompts=n,
                                       page_size=attn.desc.page_size, causal=False, sm_scale=attn.desc.sm_scale)
        sizes = (B.accumulate_kv_weights_workspace_size(self.desc, n, 1, room), B.select_kv_tokens_workspace_size(n, hkv, room))
        _require(min(sizes) > 0 and n * hkv <= B.SPD_MAX_COMPACT_ROWS, "these are more than accumulate_kv_weights, select_kv_tokens or compact_kv takes")
        self.one_each = torch.arange(n + 1, dtype=torch.int32, device=dev)
        if attn.desc.page_size:
            self.starts = attn.suffix_page_indptr
        else:
            _require(n * room < 2 ** 31, "contiguous suffixes of 2^31 tokens and more have no 32-bit starts")
            self.starts = self.one_each * room
        self.weights = torch.zeros((n, hkv, room), dtype=torch.float32, device=dev)
        self.source = torch.empty((n, hkv, budget), dtype=torch.int32, device=dev)
        self.new_lens = torch.empty(n, dtype=torch.int32, device=dev)
        self.workspace = torch.empty(max(sizes), dtype=torch.uint8, device=dev)

    def reset(self) -> None:
        self.weights.zero_()

    def accumulate(self, stream=None) -> None:
        a = self.attn
        B.accumulate_kv_weights(self.desc, a.q, a.k_suffix, self.one_each, a.suffix_lens, self.starts, a.suffix_page_indices, a.lse,
                                a.q.shape[0], 1, a.max_suffix_len, self.decay, self.weights, self.weights, self.weights.stride(1),
                                self.workspace, stream)

    def evict(self, stream=None) -> None:
        a, (n, hkv, room) = self.attn, self.weights.shape
        B.select_kv_tokens(self.weights, room, n, hkv, a.suffix_lens, room, None, self.budget, self.sinks, self.recent, self.source,
                           self.budget, self.new_lens, self.workspace, stream)
        B.compact_kv(self.desc, self.source, self.source.stride(0), self.source.stride(1), self.new_lens, self.budget, self.starts,
                     a.suffix_page_indices, a.k_suffix, a.v_suffix, self.starts, a.suffix_page_indices, a.k_suffix, a.v_suffix,
                     self.weights, self.weights, room, a.suffix_lens, stream)


class DecodeLoop:
    """A loop of decode steps on the device: append the step's K/V (synthetic: there are no
    weights), attention, sampling; lengths, finished flags and the step counter live on the
    device, so the steps can be replayed from a captured graph without host synchronisation.
    Every kernel of a step is one of the library's own launches.

    With `raw_logits` ([rows, vocab], fp32 or bf16) and `penalties` (arguments of `make_penalties` other than
    `tokens` and `token_lens`) every step shapes the raw logits by what the loop has drawn so far, into the
    sampler's own logits, before it samples (needs `one_launch`: the step's first launch records the token
    drawn before it).  How many there are follows the step counter: a loop whose counter is set back starts
    from none, whatever its record still holds.

    With `logprobs` (a DeviceLogprobs of the sampler's `tokens`) every step says how probable what it drew was:
    logprobs_steps, ranks_steps, entropy_steps [steps, rows] and top_tokens_steps, top_logprobs_steps [steps, rows, num_top].  With
    `eviction` (a DeviceEviction of `attn`) every step's attention adds to the weights of the tokens it looked at; `eviction.evict()`
    between two steps, before the suffixes are full, makes room (a full suffix takes no new token); lens_steps has what the next step finds.

    Per-step inputs are rows of tensors indexed by the device-side step counter:
      q_steps [steps, N, Hq, D], k_steps / v_steps [steps, N, Hkv, D], u_steps [steps, rows].
    The logits are the same every step (only the uniforms change); `tokens_steps`, `out_steps`
    and `lens_steps` record every step's results for checking."""

    def __init__(self, attn: DeviceAttn, sampler: DeviceSampler, q_steps, k_steps, v_steps, u_steps,
                 end_token: int = -1, one_launch: bool = True, raw_logits=None, penalties: Optional[dict] = None,
                 logprobs: Optional[DeviceLogprobs] = None, eviction: Optional[DeviceEviction] = None):
        if (raw_logits is None) != (penalties is None) or (penalties is not None and not one_launch):
            raise ValueError("raw_logits and penalties go together, and need one_launch")
        if penalties is not None:
            _check_penalties(sampler, raw_logits, penalties)
        _require(logprobs is None or logprobs.tokens is sampler.tokens, "logprobs have to be those of the sampler's tokens")
        _require(eviction is None or eviction.attn is attn, "eviction has to be that of this attention call")
        self.attn, self.sampler = attn, sampler
        self.logprobs, self.eviction = logprobs, eviction
        self.one_launch = one_launch
        self.q_steps, self.k_steps, self.v_steps, self.u_steps = q_steps, k_steps, v_steps, u_steps
        self.steps = q_steps.shape[0]
        dev = q_steps.device
        n = attn.q.shape[0]
        self.step = torch.zeros(3, dtype=torch.int64, device=dev)  # {current, next, arrivals}
        self.finished = torch.zeros(n, dtype=torch.int32, device=dev)
        self.end_token = end_token
        sampler.tokens.fill_(-1)  # "no token yet": never equal to an end token (>= 0)
        self.k_cur = torch.empty_like(k_steps[0])
        self.v_cur = torch.empty_like(v_steps[0])
        self.tokens_steps = torch.full((self.steps, sampler.tokens.shape[0]), -1, dtype=torch.int32, device=dev)
        self.out_steps = torch.zeros((self.steps,) + tuple(attn.out.shape), dtype=attn.out.dtype, device=dev)
        self.lens_steps = torch.zeros((self.steps, n), dtype=torch.int32, device=dev)
        nbytes = lambda t: t.numel() * t.element_size()
        self._select = B.make_row_copies([(q_steps, attn.q, nbytes(attn.q)), (k_steps, self.k_cur, nbytes(self.k_cur)),
                                          (v_steps, self.v_cur, nbytes(self.v_cur)),
                                          (u_steps, sampler.uniforms, nbytes(sampler.uniforms))])
        said = []  # what the log probabilities' call leaves, and where every step's goes
        if logprobs is not None:
            for name in ("logprobs", "ranks", "entropy") + (("top_tokens", "top_logprobs") if logprobs.num_top else ()):
                x = getattr(logprobs, name)
                steps = torch.zeros((self.steps,) + tuple(x.shape), dtype=x.dtype, device=dev)
                setattr(self, name + "_steps", steps)
                said.append((x, steps, nbytes(x)))
        self._record = B.make_row_copies([(sampler.tokens, self.tokens_steps, nbytes(sampler.tokens)),
                                          (attn.out, self.out_steps, nbytes(attn.out)),
                                          (attn.suffix_lens, self.lens_steps, nbytes(attn.suffix_lens))] + said)
        # one launch per step: the lengths are recorded by the append itself, K and V rows are read
        # straight from the step tensors
        self._select_qu = B.make_row_copies([(q_steps, attn.q, nbytes(attn.q)),
                                             (u_steps, sampler.uniforms, nbytes(sampler.uniforms))])
        self._record_to = B.make_row_copies([(sampler.tokens, self.tokens_steps, nbytes(sampler.tokens)),
                                             (attn.out, self.out_steps, nbytes(attn.out))] + said)
        self.raw_logits, self.penalties = raw_logits, None
        if penalties is not None:
            # one more step input: step t's history is the record's first t rows (steps past the last repeat its inputs,
            # this one too)
            rows = self.tokens_steps.shape[1]
            self._drawn = torch.zeros(rows, dtype=torch.int32, device=dev)
            self._drawn_steps = torch.arange(self.steps, dtype=torch.int32, device=dev)[:, None].repeat(1, rows)
            self._select_qu = B.make_row_copies([(q_steps, attn.q, nbytes(attn.q)),
                                                 (u_steps, sampler.uniforms, nbytes(sampler.uniforms)),
                                                 (self._drawn_steps, self._drawn, nbytes(self._drawn))])
            self._penalty_tensors = dict(penalties, tokens=self.tokens_steps.t(), token_lens=self._drawn)
            self.penalties = B.make_penalties(**self._penalty_tensors)

    def _shape_logits(self) -> None:
        raw, s = self.raw_logits, self.sampler
        B.penalize_logits(raw, B.SPD_BF16 if raw.dtype == torch.bfloat16 else B.SPD_F32, raw.shape[0], raw.shape[1], raw.stride(0),
                          self.penalties, s.logits, s.logits.stride(0))

    def _attend(self) -> None:
        self.attn.run()
        if self.eviction is not None:
            self.eviction.accumulate()

    def _sample(self) -> None:
        self.sampler.run()
        if self.logprobs is not None:
            self.logprobs.run()

    def one_step(self) -> None:
        """Enqueues one decode step on the current stream (capturable: kernel launches only).  With
        `one_launch` the results of a step are recorded by the next step's advance call, those of
        the last step by `flush`."""
        a, s = self.attn, self.sampler
        if self.one_launch:
            B.decode_step_advance(self.step, self.steps, self._record_to, self._select_qu, a.desc, self.k_steps,
                                  self.v_steps, a.k_suffix, a.v_suffix, a.suffix_lens, a.suffix_page_indptr,
                                  a.suffix_page_indices, a.max_suffix_len, s.tokens, self.end_token, self.finished,
                                  self.lens_steps)
            self._attend()
            if self.penalties is not None:
                self._shape_logits()
            self._sample()
            return
        B.decode_step_select(self.step, self.steps, self._select)
        B.append_suffix_kv(a.desc, self.k_cur, self.v_cur, a.k_suffix, a.v_suffix, a.suffix_lens,
                           a.suffix_page_indptr, a.suffix_page_indices, a.max_suffix_len,
                           s.tokens, self.end_token, self.finished)
        self._attend()
        self._sample()
        B.decode_step_record(self.step, self.steps, self._record)

    def flush(self) -> None:
        """After the last step of a `one_launch` loop: records that step's results."""
        if self.one_launch:
            B.decode_step_record(self.step, self.steps, self._record)


@dataclasses.dataclass
class DeviceLevel:
    k: torch.Tensor
    v: torch.Tensor
    lens: torch.Tensor
    indptr: torch.Tensor
    sample_indptr: torch.Tensor
    max_samples_per_group: int
    max_len: int


class DeviceCascade:
    """A CascadeInputs record on the GPU and the multi-level attention call on it."""

    def __init__(self, inp, device="cuda:0"):
        sp = inp.spec
        bf16 = sp.dtype == "bf16"
        n, hq, d = inp.q.shape
        self.desc = B.make_desc(dtype=B.SPD_BF16 if bf16 else B.SPD_F32, num_q_heads=hq,
                                num_kv_heads=sp.num_kv_heads, head_dim=d, num_prompts=1, num_samples=n)
        self.q = _dev(inp.q, device, bf16)
        self.levels = [DeviceLevel(_dev(lv.k, device, bf16), _dev(lv.v, device, bf16), _dev(lv.lens, device),
                                   _dev(lv.indptr, device), _dev(lv.sample_indptr, device),
                                   lv.max_samples_per_group, lv.max_len) for lv in inp.levels]
        self.level_array = B.make_levels(self.levels)
        self.k_suffix, self.v_suffix = _dev(inp.k_suffix, device, bf16), _dev(inp.v_suffix, device, bf16)
        self.suffix_lens = _dev(inp.suffix_lens, device)
        self.max_suffix_len = inp.max_suffix_len
        self.out = torch.empty((n, hq, d), dtype=torch.bfloat16 if bf16 else torch.float32, device=device)
        self.lse = torch.empty((n, hq), dtype=torch.float32, device=device)
        nbytes = B.shared_prefix_decode_attn_levels_workspace_size(self.desc, self.level_array, self.max_suffix_len)
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)

    def run(self, stream=None) -> None:
        B.shared_prefix_decode_attn_levels(self.desc, self.q, self.level_array, self.k_suffix, self.v_suffix,
                                           self.suffix_lens, None, None, self.max_suffix_len, self.out, self.lse,
                                           self.workspace, stream)
