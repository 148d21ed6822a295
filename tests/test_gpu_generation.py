"""The attention block of a decoder layer as generation uses it: quantized q, k and v projections, the cache, the attention, the quantized
output projection; a prompt in two pieces, then tokens one at a time, with sequences that join and leave.  Against the
same block in 64 bits that keeps every key and value."""
import math

import pytest
import torch

import oracle
from paper_2305_14152_b200 import binding
from gpu_util import dev_to_f64
from kv_util import angles

DIM, HEADS, KV = 64, 8, 2
WIDTH = HEADS * DIM


def _linears(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    made = []
    for n in (WIDTH, KV * DIM, KV * DIM, WIDTH):
        w = binding.quantize_rtn(torch.randn((n, WIDTH), generator=gen, device="cuda") / math.sqrt(WIDTH), 4, 0)
        codes = torch.from_numpy(oracle.unpack(w.qweight.cpu().numpy().view("uint32"), WIDTH, 4).astype("int64"))
        made.append((w, binding.decode_prepare(w), (codes - w.zeros.cpu().long()).double() * w.scales.cpu().double()))
    torch.cuda.synchronize()
    return made


def _turn(x, pos, cos_sin):
    c, s = cos_sin[pos, None, :DIM // 2].double(), cos_sin[pos, None, DIM // 2:].double()
    a, b = x[..., :DIM // 2], x[..., DIM // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,worst", [(torch.bfloat16, 0.03), (torch.int8, 0.06)])
def test_prompt_and_tokens(dtype, worst):
    """worst: of an output's size.  A chain of roundings, each 2^-8 of its value at most: x W, its rotation and its place in the cache, out, and the
    output projection, with q and k going through scores of size 1 into p: six of them add to 2.4 %.  int8: 1/254 of the head's largest, about
    3 rms, is 2^-6.4 of the rms at most, for k and for v beside them."""
    lin = _linears(3)
    gen = torch.Generator().manual_seed(4)
    table = torch.randperm(24, generator=gen).to(torch.int32).view(3, 8).cuda()
    cache = binding.alloc_kv_cache(24, 16, KV, DIM, table, dtype)
    cos_sin = angles(128, DIM)
    cos_gpu, ws = cos_sin.cuda(), binding.alloc_attn_workspace(cache, HEADS)
    dense = [[torch.zeros(0, KV, DIM, dtype=torch.float64)] * 2 for _ in range(3)]      # what every sequence has, in 64 bits
    lens = [0, 0, 0]

    def project(x, i):
        return binding.qlinear_fwd(lin[i][0], x) if x.shape[0] > 16 else binding.qlinear_decode_prepared(lin[i][0], lin[i][1], x)

    def remember(b, rows):
        """keys and values of new tokens in 64 bits; their rotated queries"""
        pos = torch.arange(dense[b][0].shape[0], dense[b][0].shape[0] + rows.shape[0])
        heads = lambda i: (rows.double() @ lin[i][2].t()).view(rows.shape[0], lin[i][2].shape[0] // DIM, DIM)
        dense[b] = [torch.cat([dense[b][0], _turn(heads(1), pos, cos_sin)]), torch.cat([dense[b][1], heads(2)])]
        return _turn(heads(0), pos, cos_sin)

    def append(x, counts):
        q, k, v = (project(x.cuda(), i).view(x.shape[0], -1, DIM) for i in range(3))
        for b, c in enumerate(counts):
            lens[b] += c
            remember(b, x[sum(counts[:b]):sum(counts[:b + 1])])
        starts = torch.tensor([sum(counts[:b]) for b in range(4)], dtype=torch.int32, device="cuda")
        binding.kv_append(cache, q, k, v, cos_gpu, torch.tensor(lens, dtype=torch.int32, device="cuda"), starts)

    draw = lambda n: torch.randn(n, WIDTH, generator=gen).bfloat16()
    append(draw(60), [33, 0, 27])
    append(draw(25), [7, 18, 0])
    for step in range(6):
        live = [0 if step in (2, 3) and b == 1 else 1 for b in range(3)]                # sequence 1 pauses for two steps
        x = torch.zeros(3, WIDTH, dtype=torch.bfloat16)
        x[[b for b in range(3) if live[b]]] = draw(sum(live))
        # a batch of fixed size: one row per sequence, length 0 for one that is not there
        q, k, v = (project(x.cuda(), i).view(3, -1, DIM) for i in range(3))
        for b in range(3):
            lens[b] += live[b]
        lens_gpu = torch.tensor([n * on for n, on in zip(lens, live)], dtype=torch.int32, device="cuda")
        q = binding.kv_append(cache, q, k, v, cos_gpu, lens_gpu)
        o = binding.attn_decode(cache, q, lens_gpu, workspace=ws)
        y = project(o.view(3, WIDTH), 3)
        binding.check_status()
        for b in range(3):
            if not live[b]:
                assert (q[b] == 0).all() and (o[b] == 0).all()
                continue
            turned = remember(b, x[b:b + 1])
            s = torch.einsum("kgd,tkd->kgt", turned[0].view(KV, -1, DIM), dense[b][0]) / math.sqrt(DIM)
            want = torch.einsum("kgt,tkd->kgd", s.softmax(-1), dense[b][1]).reshape(-1) @ lin[3][2].t()
            got = torch.from_numpy(dev_to_f64(y[b]))
            assert (got - want).norm() <= worst * want.norm(), (step, b, float((got - want).norm() / want.norm()))


@pytest.mark.gpu
@pytest.mark.parametrize("seqs,length", [(3, 100), (16, 900)])
def test_captured_steps_follow_one_another(seqs, length):
    """Projections, append, attention and output projection of two layers in one graph, each kernel's launch under the one before: replayed, the bits
    of the same calls one at a time.  Few rows, and more than there are CTAs."""
    lin = _linears(5)
    gen = torch.Generator().manual_seed(6)
    kv = KV if seqs < 10 else HEADS + 2                      # (the second: a cache of its own width, its keys and values not projected)
    heads = HEADS if seqs < 10 else HEADS + 2
    pages = -(-length // 16)
    tables = [torch.randperm(seqs * pages, generator=gen).to(torch.int32).view(seqs, pages).cuda() for _ in range(2)]
    caches = [binding.alloc_kv_cache(seqs * pages, 16, kv, DIM, t) for t in tables]
    for c in caches:
        for x in (c.k, c.v):
            x.copy_(torch.randn(x.shape, generator=gen).bfloat16())
    start = [(c.k.clone(), c.v.clone()) for c in caches]
    cos_sin, ws = angles(length, DIM).cuda(), binding.alloc_attn_workspace(caches[0], heads)
    x = torch.randn(seqs, WIDTH, generator=gen).bfloat16().cuda()
    lens = torch.randint(1, length + 1, (seqs,), generator=gen).to(torch.int32).cuda()
    more = torch.randn(seqs, 3, 2, DIM, generator=gen).bfloat16().cuda()

    def step(between):
        y = x
        for c in caches:
            q, k, v = (binding.qlinear_decode_prepared(lin[i][0], lin[i][1], y).view(seqs, -1, DIM) for i in range(3))
            if kv != KV:
                k, v, q = torch.cat([q, more[:, 0]], 1), torch.cat([q, more[:, 1]], 1), torch.cat([q, more[:, 2]], 1)
            between()
            q = binding.kv_append(c, q, k, v, cos_sin, lens)
            between()
            o = binding.attn_decode(c, q, lens, workspace=ws)
            between()
            y = binding.qlinear_decode_prepared(lin[3][0], lin[3][1], o[:, :HEADS].contiguous().view(seqs, WIDTH))
            between()
        return y

    want = step(torch.cuda.synchronize)
    wrote = [(c.k.clone(), c.v.clone()) for c in caches]
    step(lambda: None)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(lambda: None)
    for _ in range(3):
        for c, (k, v) in zip(caches, start):
            c.k.copy_(k)
            c.v.copy_(v)
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        for c, (k, v) in zip(caches, wrote):
            assert torch.equal(c.k, k) and torch.equal(c.v, v)
    binding.check_status()
