"""Caches held in 4 bits for the GPU tests: a host model whose rows are the
packed bytes, and the same pages on the GPU."""

import numpy as np
import torch

from oracle import evict_oracle as EO
from oracle import paged_oracle as PO
from paper_2606_01790_amd import paged as pg
from paper_2606_01790_amd import workload as WL


def bf16(x):
    """fp64 values rounded to bf16, as fp64."""
    return WL.bf16_bits_to_f32(WL.f32_to_bf16_bits(np.asarray(x, dtype=np.float32))).astype(np.float64)


def to_bf16(x):
    """fp64 values that are bf16 numbers, on the GPU."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(torch.bfloat16)


def pool_on_gpu(blocks, order="plain"):
    """Blocks [nl, n_pages, G, bytes] on the GPU: plain; the group outermost; or 32
    bytes between the blocks."""
    t = torch.from_numpy(np.ascontiguousarray(blocks)).cuda()
    if order == "groups":
        return t.permute(2, 1, 0, 3).contiguous().permute(2, 1, 0, 3)
    if order == "padded":
        return torch.cat([t, torch.full_like(t[..., :32], 255)], -1)[..., :t.shape[-1]]
    return t


def cache_of(m, H, d, order="plain"):
    """The model's pages as a cache."""
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return pg.Cache(pool_on_gpu(EO.fp4_blocks(m.k), order), pool_on_gpu(EO.fp4_blocks(m.v), order),
                    i32(m.table), i32(m.len), i32(m.refs), H, d)


def empty_model(nl, n_pages, G, P, d, n_slots, max_pages, fill=255):
    pool = np.full((nl, n_pages, G, P, EO.fp4_row_bytes(d)), fill, dtype=np.uint8)
    return PO.PagedModel(pool, pool.copy(), n_slots, max_pages)


def model_of(c):
    """The host model with what a cache holds now (rows of a plain one in fp64), and what
    makes its rows numbers."""
    if c.fp4:
        n, out = c.page_tokens * c.d // 2, []
        for t in (c.k, c.v):
            x = t.cpu().numpy()
            lead = x.shape[:3]
            out.append(np.concatenate([x[..., :n].reshape(*lead, -1, c.d // 2),
                                       x[..., n:].reshape(*lead, -1, c.d // 32)], -1))
    else:
        out = [t.double().cpu().numpy() for t in (c.k, c.v)]
    m = PO.PagedModel(*out, *c.table.shape)
    m.table, m.len, m.refs = c.table.cpu().numpy(), c.length.cpu().numpy(), c.refs.cpu().numpy()
    return m, EO.fp4_numbers if c.fp4 else lambda x: x
