"""Setups shared by the tests of the 4-bit cache and of eviction: paged pools of
random rows on the GPU beside their fp64 values, and error bounds."""
import numpy as np

import torch

from oracle import kara_cache as oc

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 2.0 ** -24          # half a step of fp32, relative


def table_for(rng, lens, bs, max_blocks, extra=5):
    """A fragmented block table that maps every sequence's tokens, and the pool's pages."""
    need = [-(-int(n) // bs) for n in lens]
    pages = sum(need) + extra
    perm = rng.permutation(pages)
    table = np.full((len(lens), max_blocks), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = perm[at:at + n]
        at += n
    return table, pages, perm[at:]


def params(Hq, Hkv, d, bs, pages, max_blocks, n_seqs, dtype, scale=0.0):
    from paper_2607_01237_amd import kara
    return kara.make_params(dict(window=64, buffer=0, budget=16, chunk_budget=4, max_chunk_len=4, head_dim=d, n_q_heads=Hq,
                                 n_kv_heads=Hkv, block_size=bs, num_pages=pages, max_blocks_per_seq=max_blocks,
                                 dtype=dtype, scale=scale), n_seqs)


def gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def random_q4(rng, shape, d):
    """Codes and scale bytes of random rows; a few far larger and smaller blocks."""
    codes = rng.integers(0, 256, shape + (d // 2,), dtype=np.uint8)
    scales = rng.integers(122, 129, shape + (d // 32,), dtype=np.uint8)
    return codes, scales


def rows_of(pool, table, s, n, bs):
    """[n, Hkv, ...] rows of sequence s from a pool [pages, Hkv, bs, ...]."""
    at = np.arange(n)
    return pool[table[s][at // bs], :, at % bs]


def logit_error(q, k, scale, terms=1):
    """How far an fp32 logit may be off, relative to its exponential, for queries q
    [.., Hq, d] over keys k [n, Hkv, d]: products of d terms summed in fp32 in any order (d EPS of the sum of magnitudes), scaled
    by a rounded constant (3 EPS of the logit: constant, product, subtraction of
    the maximum), exponentiated within 2 EPS.  `terms`: bf16 terms a factor is
    held in, 24 bits of it in three (another EPS of the magnitudes each)."""
    d = q.shape[-1]
    Hq, Hkv = q.shape[-2], k.shape[-2]
    mags = scale * max(float((np.abs(q[..., h, :]).reshape(-1, d) @ np.abs(k[:, h * Hkv // Hq]).T).max()) for h in range(Hq))
    return (d + 3 + 2 * terms) * EPS * mags + 3 * EPS


def attention_bound(out, mass, delta, n, dtype, bf16_weights):
    """|error| of an output element: every weight off by a factor 1 + 2 delta (its
    own and the sum's), n products summed in fp32 (n EPS of the mass, and as much
    for the sum), bf16 weights (half a step, 2^-8, in the numerator and in the
    sum), and the output's own rounding."""
    rel = 2 * delta + 2 * (n + 8) * EPS + (2 * 2.0 ** -8 if bf16_weights else 2 * EPS)
    return 1.05 * rel * mass + (2.0 ** -8 if dtype == "bf16" else 2 * EPS) * np.abs(out) + 1e-30
