"""Sizes and masks for each form that attention takes by its rules (row tiles
of 32 and 128, key parts, packed heads, head parts, backward in one launch and
in two), and the form each is meant for."""
import torch

from paper_2007_00072_amd import lib


def i32(*x):
    return torch.tensor(x, dtype=torch.int32)


def slopes(H):
    return torch.exp2(-torch.arange(1, H + 1).double() * 8 / H).float()


def far_documents(K):
    """Documents in pieces of 64 to 200 positions; the first keys' one goes on behind the 64th step of any form."""
    doc = torch.bucketize(torch.arange(K), torch.arange(100, K, 137)).int() + 1
    doc[:30] = 0
    doc[40:60] = -1
    doc[K - 150:K - 90] = 0
    doc[K // 2:K // 2 + 5] = 0
    doc[-1] = 0
    return doc


def case(rows, key_parts, head_parts, apart, B, J, K, H, G, P, heads=None, batches=None, grads=True, dirty=False, **kw):
    """key_parts, head_parts: whether there are several; heads, batches: those compared (all)."""
    return dict(form=(rows, key_parts, head_parts, apart), size=(B, J, K, H, G, P), heads=heads, batches=batches,
                grads=grads, dirty=dirty, kw=kw)


def cases():
    c = {}
    ragged = dict(k_len=i32(520, 0, 1, 300), q_len=i32(300, 7, 200, 300))
    doc520 = torch.stack([torch.bucketize(torch.arange(520), torch.tensor(x), right=True).int()
                          for x in ([64, 65, 300], [1, 128, 256, 511], [200], [10, 20, 30, 40, 333])])
    doc520[2, 100:180] = -1
    doc520[3, 500:] = -1
    for P in (32, 64, 96, 128):
        c[f"parts_{P}"] = case(128, True, True, False, 4, 300, 520, 8, 4, P, causal=True)
        c[f"whole_{P}"] = case(128, False, False, False, 4, 300, 400, 8, 8, P)
    for P in (40, 64):
        c[f"prefix_{P}"] = case(128, True, True, False, 4, 300, 520, 8, 4, P, causal=True, prefix=i32(0, 5, 520, 64), **ragged)
        c[f"cap_bias_{P}"] = case(128, True, True, False, 4, 300, 520, 8, 4, P, causal=True, cap=3.0, slopes=slopes(8))
        c[f"bias_{P}"] = case(128, False, False, False, 4, 300, 400, 8, 8, P, slopes=slopes(8))
        c[f"documents_{P}"] = case(128, True, True, False, 4, 520, 520, 8, 4, P, doc=doc520)
        c[f"documents_causal_{P}"] = case(128, True, True, False, 4, 300, 520, 8, 4, P, doc=doc520, causal=True,
                                          slopes=slopes(8))
        c[f"dirty_{P}"] = case(128, True, True, False, 4, 300, 520, 8, 4, P, doc=doc520, causal=True, dirty=True,
                               k_len=i32(520, 301, 400, 333), q_len=i32(300, 299, 5, 300))
    c["cap_ragged_128"] = case(128, True, True, False, 4, 300, 520, 8, 4, 128, cap=5.0, **ragged)
    # query heads of a key/value head side by side in tiles of 128
    c["packed"] = case(128, True, True, False, 8, 100, 1200, 8, 2, 64, causal=True, slopes=slopes(8))
    c["packed_documents"] = case(128, True, True, False, 8, 100, 1200, 8, 2, 32, causal=True,
                                 doc=far_documents(1200).expand(8, 1200).contiguous(), k_len=i32(*range(1200, 400, -100)))
    # a chunk behind a long cache, few heads: many parts
    c["chunk"] = case(128, True, True, False, 2, 200, 4100, 4, 1, 64, causal=True, k_len=i32(4100, 1234))
    c["chunk_documents"] = case(128, True, True, False, 2, 200, 4100, 4, 1, 96, causal=True, k_len=i32(4100, 3000),
                                doc=torch.stack([far_documents(4100), torch.zeros(4100, dtype=torch.int32)]))
    # more than 64 steps a block, forward and backward
    for P in (32, 96):
        c[f"windows_{P}"] = case(128, False, False, P > 64, 1, 4300, 4300, 12, 12, P, heads=(0, 11),
                                 doc=far_documents(4300)[None].contiguous())
    c["windows_causal"] = case(128, False, False, False, 1, 4300, 4300, 12, 12, 64, heads=(5,), causal=True,
                               doc=far_documents(4300)[None].contiguous(), k_len=i32(4299), q_len=i32(4250))
    c["windows_few"] = case(32, False, False, False, 64, 1, 9000, 16, 16, 8, heads=(0, 15), batches=(0, 63), grads=False,
                            doc=far_documents(9000).expand(64, 9000).contiguous())
    c["few_parts"] = case(32, True, True, False, 2, 1, 9000, 8, 2, 64, causal=True, k_len=i32(9000, 7000),
                          doc=torch.stack([far_documents(9000), torch.zeros(9000, dtype=torch.int32)]))
    return c


def desc(size, doc=False, **kw):
    B, J, K, H, G, P = size
    d = lib.AttnDesc(B, J, K, H, G, P, lib.DM_BF16, 0.0, 0.0, 1 if kw.get("causal") else 0)
    d.q = d.out = lib.AttnStride(J * H * P, P, H * P)
    d.k = d.v = lib.AttnStride(K * G * P, P, G * P)
    return d
