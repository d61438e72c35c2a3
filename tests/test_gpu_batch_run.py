"""The operators of include/spec_batch.h in a row, as a program runs a verification pass with them: eager, captured, on streams
of their own, and in a process whose first calls are captured.

Tolerance of the run in fp32: keys and queries are off by 3 * 2^-24 of their terms (the rotation), so scores by 8 * 2^-24 A more
than the attention's own bound, A = scale sum |q k|; everything else as in test_gpu_batch.py."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import batch_reference as ref
import paper_2504_00030_amd as pk

pytestmark = pytest.mark.gpu

B, NQ, NKV, HD, ROT, PAGE, PREFIX, V = 3, 4, 2, 64, 48, 16, 37, 500
DRAFTS = [2, 0, 3]
HISTORY = [20, 1, 40]  # own positions in front of this pass's rows
ROWS = [k + 1 for k in DRAFTS]
R, D = sum(ROWS), sum(DRAFTS)
WIDTH = (NQ + 2 * NKV) * HD


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


class Pass:
    def __init__(self, seed, dtype):
        rng = np.random.default_rng(seed)
        self.rng, self.dtype = rng, dtype
        own = [h + n for h, n in zip(HISTORY, ROWS)]
        n_own = (max(own) + PAGE - 1) // PAGE
        n_prefix = (PREFIX + PAGE - 1) // PAGE
        perm = rng.permutation(n_prefix + B * n_own)
        self.prefix_table, self.table, self.own = perm[:n_prefix], perm[n_prefix:].reshape(B, n_own), own
        slot = lambda table, j: int(table[j // PAGE]) * PAGE + j % PAGE
        self.cos, self.sin = (torch.zeros((256, ROT // 2), device="cuda") for _ in range(2))
        self.k, self.v = (torch.full((len(perm), NKV, PAGE, HD), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
        # the prefix, and what the sequences hold already, as rows of their own
        self.before = rng.standard_normal((PREFIX + sum(HISTORY), WIDTH)).astype(np.float32)
        self.before_pos = list(range(PREFIX)) + [PREFIX + j for h in HISTORY for j in range(h)]
        self.before_slot = [slot(self.prefix_table, j) for j in range(PREFIX)] + [slot(self.table[b], j) for b in range(B) for j in range(HISTORY[b])]
        self.pos = [PREFIX + HISTORY[b] + i for b in range(B) for i in range(ROWS[b])]
        self.slot = [slot(self.table[b], HISTORY[b] + i) for b in range(B) for i in range(ROWS[b])]
        self.rows = torch.from_numpy(rng.standard_normal((R, WIDTH)).astype(np.float32)).to(dtype).cuda()
        self.head = torch.from_numpy((rng.standard_normal((NQ * HD, V)) * 0.3).astype(np.float32)).cuda()
        self.q_out, self.out = (torch.zeros((R, NQ, HD), dtype=dtype, device="cuda") for _ in range(2))
        self.p, self.q = torch.zeros((R, V), device="cuda"), torch.softmax(torch.from_numpy(rng.standard_normal((D, V)).astype(np.float32)).cuda(), 1)
        self.drafted = _i32(rng.integers(0, V, D))
        self.ua, self.un = (torch.from_numpy(rng.random(n).astype(np.float32)).cuda() for n in (D, B))
        self.A, self.y = _i32([9] * B), _i32([9] * B)
        starts = lambda n: np.concatenate([[0], np.cumsum(n)])
        self.row_start, self.draft_start = _i32(starts(ROWS)), _i32(starts(DRAFTS))
        self.d_pos, self.d_slot, self.d_table, self.d_own, self.d_prefix = _i32(self.pos), _i32(self.slot), _i32(self.table), _i32(own), _i32(self.prefix_table)
        n = pk.k_attn_shared_workspace(R, B, NQ, NKV, HD, dtype, PREFIX, n_own * PAGE)
        self.attn_work = torch.full((max(n, 16),), 0xff, dtype=torch.uint8, device="cuda")
        self.verify_work = torch.full((pk.k_verify_workspace(B, V),), 0xff, dtype=torch.uint8, device="cuda")

    @staticmethod
    def heads(rows):
        return (rows[:, : NQ * HD].unflatten(1, (NQ, HD)), rows[:, NQ * HD: (NQ + NKV) * HD].unflatten(1, (NKV, HD)),
                rows[:, (NQ + NKV) * HD:].unflatten(1, (NKV, HD)))

    def fill(self):
        s = torch.cuda.current_stream().cuda_stream
        pk.k_rope_tables(self.cos, self.sin, theta=500000.0, scaling="bands", factor=8.0, low=1.0, high=4.0, context=64.0, stream=s)
        _, k, v = self.heads(torch.from_numpy(self.before).to(self.dtype).cuda())
        pk.k_rope_cache(None, k, v, self.cos, self.sin, _i32(self.before_pos), _i32(self.before_slot), None, self.k, self.v, stream=s)

    def step(self):
        s = torch.cuda.current_stream().cuda_stream
        q, k, v = self.heads(self.rows)
        pk.k_rope_cache(q, k, v, self.cos, self.sin, self.d_pos, self.d_slot, self.q_out, self.k, self.v, stream=s)
        pk.k_attn_shared(self.q_out, self.k, self.v, self.row_start, self.d_table, self.d_own, self.out, self.attn_work, prefix_table=self.d_prefix,
                         prefix_len=PREFIX, stream=s)
        torch.softmax(self.out.float().flatten(1) @ self.head, 1, out=self.p)
        pk.k_verify(self.p, self.q, self.draft_start, self.drafted, self.ua, self.un, self.A, self.y, self.verify_work, stream=s)

    def results(self):
        return [t.clone() for t in (self.q_out, self.out, self.p, self.A, self.y, torch.nan_to_num(self.k), torch.nan_to_num(self.v))]


def test_a_pass_against_the_definitions():
    a = Pass(0, torch.float32)
    a.fill()
    a.step()
    torch.cuda.synchronize()
    f, _ = ref.frequencies(ROT, 500000.0, scaling="bands", factor=8.0, low=1.0, high=4.0, context=64.0)
    turn = lambda h, pos: ref.rotate(h, np.cos(np.outer(pos, f)), np.sin(np.outer(pos, f)), False)[0]
    k = np.zeros((a.k.shape[0], NKV, PAGE, HD))
    v = k.copy()
    both = np.concatenate([a.before, a.rows.double().cpu().numpy()]).astype(np.float64)
    pos, slot = np.array(a.before_pos + a.pos), np.array(a.before_slot + a.slot)
    k[slot // PAGE, :, slot % PAGE] = turn(both[:, NQ * HD: (NQ + NKV) * HD].reshape(-1, NKV, HD), pos)
    v[slot // PAGE, :, slot % PAGE] = both[:, (NQ + NKV) * HD:].reshape(-1, NKV, HD)
    q = turn(both[-R:, : NQ * HD].reshape(R, NQ, HD), np.array(a.pos))
    want, mag, n, size = ref.attention(q, k, v, np.concatenate([[0], np.cumsum(ROWS)]), a.table, a.own, a.prefix_table, PREFIX, HD ** -0.5, np.zeros(q.shape))
    rel = 2 * ((HD + 12) * size + 1) * 2.0 ** -23 + (4 * n + 16) * 2.0 ** -23
    assert (np.abs(a.out.double().cpu().numpy() - want) <= rel * mag + 2.0 ** -24 * np.abs(want)).all()
    A, y = ref.verify(a.p.double().cpu().numpy(), a.q.double().cpu().numpy(), a.draft_start.cpu().numpy(), a.drafted.cpu().numpy(),
                      a.ua.cpu().numpy(), a.un.cpu().numpy())
    assert a.A.tolist() == A.tolist() and a.y.tolist() == y.tolist()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_captured_passes_replay_on_new_inputs(dtype):
    a = Pass(1, dtype)
    a.fill()
    a.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for i in range(4):
        rng = np.random.default_rng(50 + i)
        a.rows.copy_(torch.from_numpy(rng.standard_normal((R, WIDTH)).astype(np.float32)))
        a.ua.copy_(torch.from_numpy(rng.random(D).astype(np.float32)))
        a.un.copy_(torch.from_numpy(rng.random(B).astype(np.float32)))
        if i == 2:  # lengths live in device memory: a shorter first sequence, its rows fewer positions back
            a.d_own[0] -= 7
        a.step()
        torch.cuda.synchronize()
        want = a.results()
        for t in (a.q_out, a.out, a.p, a.A, a.y):
            t.zero_()
        a.attn_work.fill_(0x7f)
        torch.randn(1 << 18, device="cuda").sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, u) for t, u in zip(a.results(), want))


def test_passes_on_two_streams_with_workspaces_of_their_own():
    """Two captured passes over different data replayed side by side, each with its buffers."""
    passes, graphs, want, streams = [Pass(2, torch.bfloat16), Pass(3, torch.bfloat16)], [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for a in passes:
        a.fill()
        a.step()
        torch.cuda.synchronize()
        want.append(a.results())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            a.step()
        graphs.append(g)
    for i in range(5):
        for a in passes:
            a.out.zero_()
            a.y.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for a, w in zip(passes, want):
            assert all(torch.equal(t, u) for t, u in zip(a.results(), w))


@pytest.mark.parametrize("rows", [3, 100])
def test_caches_beyond_32_bit_offsets(rows):
    """Pools of more than 2^31 elements: pages at their ends hold what pages of a small pool hold, and attention reads the same."""
    page, nkv, hd, n = 64, 8, 128, 150
    s = torch.cuda.current_stream().cuda_stream
    gen = torch.Generator(device="cuda").manual_seed(3)
    qkv = torch.randn((n, (8 + 2 * nkv) * hd), generator=gen, device="cuda").to(torch.bfloat16)
    q, k, v = qkv[:, : 8 * hd].unflatten(1, (8, hd)), qkv[:, 8 * hd: 16 * hd].unflatten(1, (nkv, hd)), qkv[:, 16 * hd:].unflatten(1, (nkv, hd))
    cos, sin = torch.rand((n, hd // 2), generator=gen, device="cuda"), torch.rand((n, hd // 2), generator=gen, device="cuda")
    got = []
    for n_pages in (5, 34000):
        pools = [torch.empty((n_pages, nkv, page, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        assert n_pages == 5 or pools[0].numel() > 2**31
        table = [n_pages - 1, n_pages - 3, n_pages - 2]
        slot = _i32([table[j // page] * page + j % page for j in range(n)])
        out, qo = torch.zeros((rows, 8, hd), dtype=torch.bfloat16, device="cuda"), torch.zeros((n, 8, hd), dtype=torch.bfloat16, device="cuda")
        pk.k_rope_cache(q, k, v, cos, sin, _i32(range(n)), slot, qo, *pools, stream=s)
        work = torch.empty(max(1, pk.k_attn_shared_workspace(rows, 1, 8, nkv, hd, torch.bfloat16, page, 2 * page)), dtype=torch.uint8, device="cuda")
        pk.k_attn_shared(qo[-rows:], *pools, _i32([0, rows]), _i32([table[1:]]), _i32([n - page]), out, work, prefix_table=_i32(table[:1]),
                         prefix_len=page, stream=s)
        torch.cuda.synchronize()
        got.append((qo, out, *[p[table].clone() for p in pools]))
        del pools
    places = torch.arange(3 * page, device="cuda") < n  # (places behind the last position were never written)
    for i, (a, b) in enumerate(zip(*got)):
        if i < 2:
            assert a.any() and torch.equal(a, b)
        else:
            assert torch.equal(a.transpose(1, 2).flatten(0, 1)[places], b.transpose(1, 2).flatten(0, 1)[places])


CHILD = """
import sys
sys.path.insert(0, "tests")
import torch
import test_gpu_batch_run as t
a = t.Pass(7, torch.bfloat16)
before = t._i32(a.before_pos), t._i32(a.before_slot), torch.from_numpy(a.before).to(torch.bfloat16).cuda()
def all_of_it():
    s = torch.cuda.current_stream().cuda_stream
    t.pk.k_rope_tables(a.cos, a.sin, theta=500000.0, stream=s)
    _, k, v = a.heads(before[2])
    t.pk.k_rope_cache(None, k, v, a.cos, a.sin, before[0], before[1], None, a.k, a.v, stream=s)
    q, k, v = a.heads(a.rows)
    t.pk.k_rope_cache(q, k, v, a.cos, a.sin, a.d_pos, a.d_slot, a.q_out, a.k, a.v, stream=s)
    t.pk.k_attn_shared(a.q_out, a.k, a.v, a.row_start, a.d_table, a.d_own, a.out, a.attn_work, prefix_table=a.d_prefix, prefix_len=t.PREFIX, stream=s)
    t.pk.k_verify(a.p, a.q, a.draft_start, a.drafted, a.ua, a.un, a.A, a.y, a.verify_work, stream=s)
a.p.copy_(torch.softmax(torch.randn((t.R, t.V), device="cuda"), 1))
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    all_of_it()
assert not a.out.any() and not a.cos.any() and a.A.tolist() == [9] * t.B, "a captured call ran"
all_of_it()
torch.cuda.synchronize()
want = a.results()
for i in range(3):
    for x in (a.cos, a.sin, a.q_out, a.out, a.A, a.y, a.k, a.v):
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert a.out.any() and all(torch.equal(x, y) for x, y in zip(a.results(), want))
    torch.randn(1 << 18, device="cuda").sum().item()
print("captured first")
"""


def test_first_calls_under_capture():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, PYTHONPATH=root)
    r = subprocess.run([sys.executable, "-c", CHILD], cwd=root, env=env, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "captured first" in r.stdout, r.stdout + r.stderr
