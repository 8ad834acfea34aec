"""Calls of a decoding loop one right after another on one stream, as a server makes
them: each reads what the call before it wrote, while their kernels start early."""

import pytest
import torch

from paper_2605_30351_gb300 import videomla as V

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    V.load()
    V.mla_device_status(clear=True)
    yield
    assert V.mla_device_status(clear=True) == V.MLA_OK


@pytest.mark.parametrize("new,heads", [(1, 12), (3, 12)])    # both attention kernels
def test_back_to_back_steps(new, heads):
    """40 steps of 12 streams: lengths, append, rotation in place, attention; every
    tenth step the last stream ends and becomes a branch of another one. The same
    bits without a wait as with one after every call."""
    seqs, steps, d_c, d_r = 12, 40, 192, 32
    g = torch.Generator().manual_seed(new)
    total = seqs * new

    def draw(*shape):
        return torch.randn(shape, generator=g).to(torch.bfloat16).cuda()

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    c_new, kr_new = draw(steps, total, d_c), draw(steps, total, d_r)
    q_c, q_r = draw(steps, total, heads, d_c), draw(steps, total, heads, d_r)
    pos = torch.randint(0, 500, (steps, total, 1), generator=g, dtype=torch.int32).cuda()
    q_start = ints([new * s for s in range(seqs + 1)])
    rope = V.Rope(torch.from_numpy(V.mla_rope_scaled_table_fill(d_r, 500)).cuda(),
                  (d_r // 2, 0, 0))
    lens, plan = [7 * s for s in range(seqs)], []
    start = ints(lens)
    for k in range(steps):
        branch = k % 10 == 9
        if branch:
            lens[-1] = lens[k % (seqs - 1)]
        lens = [n + new for n in lens]
        plan.append((branch, ints([k % (seqs - 1)]), ints([seqs - 1]),
                     ints([-1] * (seqs - 1) + [0]), ints(lens)))

    def run(wait):
        cache = V.PagedCache.empty(1, 400, 8, seqs, 40, d_c, d_r)
        workspace = torch.empty(V.mla_paged_workspace_bytes(cache), dtype=torch.uint8,
                                device="cuda")
        out, turned = torch.empty_like(q_c), q_r.clone()
        done = torch.cuda.synchronize if wait else (lambda: None)
        torch.cuda.synchronize()
        V.mla_pages_resize(cache, start)
        done()
        for k, (branch, src, dst, drop, grow) in enumerate(plan):
            if branch:
                V.mla_pages_resize(cache, drop)
                done()
                V.mla_pages_fork(cache, src, dst)
                done()
            V.mla_pages_resize(cache, grow)
            done()
            V.mla_paged_append(cache, 0, c_new[k], kr_new[k], q_start, pos[k], rope)
            done()
            V.mla_rope_apply(rope, turned[k], pos[k], turned[k])
            done()
            V.mla_paged_attention(cache, 0, q_c[k], turned[k], q_start, 128, 1, workspace, out[k])
            done()
        torch.cuda.synchronize()
        assert V.mla_device_status(clear=True) == V.MLA_OK
        return out, cache.table, cache.lens, cache.refs, cache.c, cache.kr

    ref = run(True)
    for _ in range(3):
        for a, b in zip(run(False), ref):
            assert torch.equal(a, b)
