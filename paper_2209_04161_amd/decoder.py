"""A transformer decoder of the library's layers: trained with approximate products, served in 8 bits.

``Decoder`` is the model in training: its dense layers are AMLinear, every product of theirs, forward and
backward, the simulated multiplier's; norms, attention and activations are exact FP32 operations, as the
paper keeps everything but the products of dense and convolution layers.  ``Decoder8`` holds the same
weights for inference in the arithmetic that an approximate multiplier is weighed against: products of 8-bit
integers, and attention over a paged cache held in 8 bits (``PagedCache8``).

    model = Decoder(2, width=256, heads=8, kv_heads=2, hidden=512, lut=lut, m_bits=7)
    y = model(x)                                     # [tokens, width], one sequence, with gradients
    served = Decoder8(model)
    cache = served.cache(pages=64)
    a, b = cache.add(), cache.add()
    y = served(x, cache, cache.extend([(a, 100), (b, 28)]))   # prompts: 100 + 28 rows of x
    y = served(x1, cache, cache.extend([(a, 1), (b, 1)]))     # then a token of each
"""
import collections

import torch

from . import binding, modules

Batch = collections.namedtuple("Batch", "page_table lengths starts max_new max_len")


def split_heads(qkv, heads, kv_heads, head_dim):
    """(q, k, v), each [tokens, heads, head_dim], views of the projection's rows."""
    h, g, d = heads, kv_heads, head_dim
    return (qkv[:, :h * d].unflatten(1, (h, d)), qkv[:, h * d:(h + g) * d].unflatten(1, (g, d)),
            qkv[:, (h + g) * d:].unflatten(1, (g, d)))


class DecoderBlock(torch.nn.Module):
    """Norm, causal attention, norm, feed-forward (ReLU); the residual's addition is part of the norms."""

    def __init__(self, width, heads, kv_heads, hidden, lut, m_bits, head_dim=None):
        super().__init__()
        if heads % kv_heads:
            raise ValueError("heads must be a multiple of kv_heads")
        self.heads, self.kv_heads = heads, kv_heads
        self.head_dim = head_dim or width // heads
        d = self.head_dim
        self.norm1 = modules.RMSNorm(width, device=lut.device)
        self.qkv = modules.AMLinear(width, (heads + 2 * kv_heads) * d, lut, m_bits, bias=False)
        self.out = modules.AMLinear(heads * d, width, lut, m_bits, bias=False)
        self.norm2 = modules.RMSNorm(width, device=lut.device)
        self.up = modules.AMLinear(width, hidden, lut, m_bits)
        self.down = modules.AMLinear(hidden, width, lut, m_bits)

    def split(self, qkv):
        return split_heads(qkv, self.heads, self.kv_heads, self.head_dim)

    def forward(self, x, residual=None):
        """(the block's output, the residual stream it is to be added to)"""
        if residual is None:
            y, h = self.norm1(x), x
        else:
            y, h = self.norm1(x, residual)
        q, k, v = (t.transpose(0, 1) for t in self.split(self.qkv(y)))
        k, v = (t.repeat_interleave(self.heads // self.kv_heads, 0) for t in (k, v))
        score = torch.matmul(q, k.transpose(1, 2).contiguous()) * self.head_dim ** -0.5
        n = x.shape[0]
        score = score.masked_fill(torch.ones((n, n), dtype=torch.bool, device=x.device).triu(1), float("-inf"))
        o = torch.matmul(torch.softmax(score, -1), v.contiguous()).transpose(0, 1).flatten(1)
        y, h = self.norm2(self.out(o), h)
        return self.down(torch.relu(self.up(y))), h


class Decoder(torch.nn.Module):
    def __init__(self, blocks, width, heads, kv_heads, hidden, lut, m_bits, head_dim=None):
        super().__init__()
        if blocks < 1:
            raise ValueError("a decoder has one block at least")
        self.blocks = torch.nn.ModuleList(
            [DecoderBlock(width, heads, kv_heads, hidden, lut, m_bits, head_dim) for _ in range(blocks)])
        self.norm = modules.RMSNorm(width, device=lut.device)

    def forward(self, x):
        """x [tokens, width]: the embedded tokens of one sequence; the normed output, [tokens, width]."""
        h = None
        for block in self.blocks:
            x, h = block(x, h)
        return self.norm(x, h)[0]


class PagedCache8:
    """Keys and values of sequences in 8 bits, for each layer (`layers`: Cache8), in pages that are handed out as the
    sequences grow.  The bookkeeping is on the host; extend() uploads what the calls need of it."""

    def __init__(self, layers, pages, heads, head_dim, page_tokens=64, device="cuda"):
        def pool(*shape, dtype=torch.int8):
            return torch.zeros(shape, dtype=dtype, device=device)

        self.page_tokens, self.device = page_tokens, device
        self.layers = [binding.Cache8(pool(pages, heads, page_tokens, head_dim), pool(pages, heads, head_dim, page_tokens),
                                      pool(pages, heads, dtype=torch.float32), pool(pages, heads, dtype=torch.float32))
                       for _ in range(layers)]
        self._free = list(range(pages - 1, -1, -1))
        self._held = {}     # sequence -> its pages
        self._lengths = {}  # sequence -> its tokens
        self._next = 0

    def add(self):
        """A new, empty sequence's number."""
        self._held[self._next], self._lengths[self._next] = [], 0
        self._next += 1
        return self._next - 1

    def release(self, sequence):
        """Gives the sequence's pages back."""
        self._free.extend(reversed(self._held.pop(sequence)))
        del self._lengths[sequence]

    def length(self, sequence):
        return self._lengths[sequence]

    def extend(self, counts):
        """Makes room for new tokens: counts is a list of (sequence, tokens); the Batch of the calls that write and
        read them, rows in the list's order.  Raises RuntimeError, and takes nothing, if pages run out."""
        if len({s for s, _ in counts}) != len(counts) or any(n < 0 for _, n in counts):
            raise ValueError("each sequence once, with a count that is not negative")
        page = self.page_tokens
        need = [max(0, -(-(self._lengths[s] + n) // page) - len(self._held[s])) for s, n in counts]
        if sum(need) > len(self._free):
            raise RuntimeError("the cache has %d free pages, the call needs %d" % (len(self._free), sum(need)))
        starts = [0]
        for (s, n), more in zip(counts, need):
            self._held[s].extend(self._free.pop() for _ in range(more))
            self._lengths[s] += n
            starts.append(starts[-1] + n)
        held = [self._held[s] for s, _ in counts]
        cols = max([len(p) for p in held] + [1])
        ints = dict(dtype=torch.int32, device=self.device)
        lengths = [self._lengths[s] for s, _ in counts]
        table = torch.tensor([p + [0] * (cols - len(p)) for p in held], **ints).reshape(len(counts), cols)
        return Batch(table, torch.tensor(lengths, **ints), torch.tensor(starts, **ints),
                     max([n for _, n in counts] + [0]), max(lengths + [0]))


def _frozen(norm):
    """The norm as it is now, without gradients."""
    weight = norm.weight.detach().clone()
    new = modules.RMSNorm(weight.numel(), norm.eps, weight.device)
    new.weight = torch.nn.Parameter(weight, requires_grad=False)
    return new


class DecoderBlock8(torch.nn.Module):
    """A DecoderBlock's weights as they are now in 8 bits, with a cache in 8 bits."""

    def __init__(self, block):
        super().__init__()
        self.heads, self.kv_heads, self.head_dim = block.heads, block.kv_heads, block.head_dim
        self.norm1, self.norm2 = _frozen(block.norm1), _frozen(block.norm2)
        self.qkv, self.out, self.up, self.down = (modules.Linear8(layer.weight, layer.bias)
                                                  for layer in (block.qkv, block.out, block.up, block.down))

    def forward(self, x, residual, cache, batch):
        """(the block's output, the residual stream); cache: this layer's Cache8."""
        y, h = self.norm1.quantized(x, residual)
        q, k, v = split_heads(self.qkv(y, x.dtype), self.heads, self.kv_heads, self.head_dim)
        table, lengths, starts, max_new, max_len = batch
        binding.amsim_cache_append(cache, table, lengths, k, v, starts, max_new)
        o = binding.amsim_cache_attention(cache, table, lengths, q, starts, max_new, max_len)
        y, h = self.norm2.quantized(self.out(o.flatten(1)), h)
        return self.down(torch.relu(self.up(y, x.dtype))), h


class Decoder8(torch.nn.Module):
    """A Decoder's weights as they are now in 8 bits, for inference.  Nothing is shared with the Decoder: it can be trained
    on, or given up."""

    def __init__(self, model):
        super().__init__()
        self.blocks = torch.nn.ModuleList([DecoderBlock8(b) for b in model.blocks])
        self.norm = _frozen(model.norm)

    def cache(self, pages, page_tokens=64):
        b = self.blocks[0]
        return PagedCache8(len(self.blocks), pages, b.kv_heads, b.head_dim, page_tokens, b.qkv.weight.device)

    @torch.no_grad()
    def forward(self, x, cache, batch):
        """x [tokens, width], float32, bfloat16 or float16: the embedded new tokens of the batch's sequences."""
        h = None
        for block, layer in zip(self.blocks, cache.layers):
            x, h = block(x, h, layer, batch)
        return binding.amsim_rmsnorm_fwd(x, self.norm.weight.detach(), self.norm.eps, residual=h).y
