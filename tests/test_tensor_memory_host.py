"""Kernels that find themselves on one SM fit into its 512 columns of tensor memory (no GPU needed: from the plans).

A CTA that has to wait for columns holds its cluster up.  If the cluster of the CTA that has them waits, on another SM, for columns of the first one (two
streams, or a launch that began early), neither ends.  Shared memory is what keeps such CTAs apart.
"""
import itertools
import re

from paper_2511_19438_b200 import build as libbuild

libbuild.build()
from paper_2511_19438_b200 import binding as B  # noqa: E402

SM_BYTES, CTA_BYTES = 228 * 1024, 1024      # shared memory of an SM, and what each CTA takes of it beside its own


def residents():
    """{(kernel, columns): the least bytes of a CTA} over sizes and types of layers."""
    least = {}

    def add(name, columns, nbytes):
        least[name, columns] = min(nbytes, least.get((name, columns), SM_BYTES))

    rows = (1, 2, 17, 32, 33, 48, 64, 65, 96, 128, 129, 200, 256, 300, 1000, 4096)
    for K, N, M in itertools.product((128, 256, 512, 1024, 2048, 4096, 11008), (128, 256, 1024, 4096, 12288, 22016), rows):
        for group in (32, 128):
            st, p = B.gptq_plan(M, N, K, group, 0, 148)
            if st == B.GPTQ_OK and p.kernel == 2:      # accumulators of a tile's tokens, 32 columns per stage of the weights
                tok = p.m_tile
                need = (2 if tok == 64 else 1) * tok + 32 * (4 if tok >= 64 else 3)
                add("tiles", 1 << (need - 1).bit_length(), p.smem_bytes)
            st, p = B.gptq_plan_decode(M, N, K, group, 0, 148)
            if st == B.GPTQ_OK:
                add("decode", 256, p.smem_bytes)
            for eight in (0, 1):
                st, p = B.gptq_plan_prefill(M, N, K, group, 0, eight, 148)
                if st == B.GPTQ_OK:
                    add("persistent", 512, p.smem_bytes)
        for gated in (0, 1):
            st, p = B.gptq_plan_fp8(M, N, K, gated, 148)
            if st != B.GPTQ_OK:
                continue
            name = p.kernel_name.decode()
            if p.kernel == 7:
                add(name, 512, p.smem_bytes)
            else:
                kind, tokens = (int(v) for v in re.findall(r"\d+", name.split("<")[1]))
                each = (1 + kind) * tokens
                add(name, max(32, each * (4 if each <= 128 else 2)), p.smem_bytes)
    return [(*k, v) for k, v in least.items()]


def test_what_shares_an_sm_fits_into_its_tensor_memory():
    all_of_them = residents()
    assert {n for n, _, _ in all_of_them} >= {"tiles", "decode", "persistent"} and len(all_of_them) >= 12
    for n in (1, 2, 3, 4):
        for together in itertools.combinations_with_replacement(all_of_them, n):
            if sum(b + CTA_BYTES for _, _, b in together) <= SM_BYTES:
                assert sum(c for _, c, _ in together) <= 512, together
