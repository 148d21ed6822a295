"""Which warp writes the list of a CTA's parts of rows (s_head of the attention kernel).  Between its first values and the parts that the warps
note there no barrier stands in every form of the kernel (few sequences, pages that end within tiles), so a warp may write its own two
entries alone.  Another warp's late store cannot be provoked from outside: the source is checked, and on a GPU the forms without a barrier
are run again and again."""
import os
import re

import pytest
import torch

from paper_2305_14152_b200 import binding
from kv_util import Case, assert_within

SOURCE = os.path.join(os.path.dirname(os.path.abspath(binding.__file__)), "csrc", "attn_decode.cu")


def test_a_warp_writes_its_own_entries_alone():
    text = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    stores = re.findall(r"\bs_head\[([^\]]*)\]\s*=(?!=)", text)
    assert len(stores) == 2, stores                        # the first values, and a part
    for index in stores:
        assert re.match(r"2 \* warp \+ (lane$|\(more)", index.strip()), index
    before = text[:text.index("s_head[2 * warp + lane]")]
    assert before.rstrip().endswith("if (lane < 2)")       # of the two that it has
    behind = text[text.index("s_head[2 * warp + lane]"):]
    assert behind[behind.index(";") + 1:].lstrip().startswith("__syncwarp();")


# (16 sequences: rows dealt out; 3: a CTA for every row; all with pages that end within tiles, or lines that lie apart)
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,dim,page_size,order", [(torch.bfloat16, 64, 16, "tokens"), (torch.int8, 128, 16, "tokens"), (torch.bfloat16, 128, 24, "heads")])
@pytest.mark.parametrize("seqs", [3, 16])
def test_no_part_is_lost_in_many_calls(dtype, dim, page_size, order, seqs):
    """One tile for most warps: the shortest way from the first values to a part."""
    case = Case(seqs + dim, [1 + (53 * i + 90) % 290 for i in range(seqs)], 16, 8 if seqs == 3 else 16, dim, page_size, dtype, order)
    cache, q, lens = case.on_gpu(), case.q.cuda(), case.lens()
    first, lse = binding.attn_decode(cache, q, lens, return_lse=True)
    ref, ref_lse, tol, lse_tol = case.attention()
    assert_within(first, ref, tol, "out")
    assert_within(lse, ref_lse, lse_tol, "lse")
    out, wrong = torch.empty_like(first), torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(2000):
        out.fill_(float("nan"))
        binding.attn_decode(cache, q, lens, out=out)
        wrong += (out.view(torch.int16) != first.view(torch.int16)).sum()
    assert int(wrong) == 0
    binding.check_status()
