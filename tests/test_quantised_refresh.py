"""Host side of the boundary refresh in 8 bits with two CPU processes over gloo: record sizes, split sizes and routing.  The cache and
its movers are stand-ins that keep a record per row (the kernels are covered on the GPU)."""
import os
import socket
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = r"""
import os, sys, numpy as np, torch, torch.distributed as dist
sys.path.insert(0, %r)
from oracle import refresh as orf
from paper_2608_16305_b200 import distributed as D
rank = int(os.environ["RANK"])
dist.init_process_group("gloo", rank=rank, world_size=2, init_method="tcp://127.0.0.1:" + os.environ["PORT"])
rng = np.random.default_rng(5)                       # same tables on both ranks
P, N, d, Q = 2, 80, 300, 3
owner = rng.integers(0, P, N)
mem = [rng.standard_normal((N, d)).astype(np.float32) for _ in range(P)]
lu = [rng.random(N) * 50 for _ in range(P)]
sets = [[sorted(rng.choice(np.nonzero(owner != p)[0], 5 + 3 * q + p, replace=False).tolist()) for p in range(P)] for q in range(Q)]
cap = max(sum(len(s) for s in sets[q]) for q in range(Q))
rn, sn = np.zeros((Q, cap), np.int32), np.zeros((Q, cap), np.int32)
ro, so = np.zeros((Q, P + 1), np.int64), np.zeros((Q, P + 1), np.int64)
for q in range(Q):
    plan = orf.refresh_plan(sets[q], owner)
    r_list, s_list = [plan[o][rank] for o in range(P)], [plan[rank][r] for r in range(P)]
    ro[q, 1:], so[q, 1:] = np.cumsum([len(x) for x in r_list]), np.cumsum([len(x) for x in s_list])
    rn[q, :ro[q, -1]], sn[q, :so[q, -1]] = sum(r_list, []), sum(s_list, [])
plan = D.RefreshPlan.from_lists(torch.from_numpy(rn), ro, torch.from_numpy(sn), so, P, rank)

class Cache:
    def __init__(self, rows, heads, dim, bits, device, record):
        assert record and rows == cap and heads == 3 and dim == 100 and bits == 8
        self.data = torch.zeros((rows, 4 * d + 8), dtype=torch.uint8)

def write(cache, memory, status, src, times):
    n = src.numel()
    cache.data[:n, :4 * d] = memory[src.long()].view(torch.uint8).view(n, 4 * d)
    cache.data[:n, 4 * d:] = times[src.long()].view(torch.uint8).view(n, 8)

def read(cache, memory, status, dst, times):
    n = dst.numel()
    memory[dst.long()] = cache.data[:n, :4 * d].contiguous().view(torch.float32).view(n, d)
    times[dst.long()] = cache.data[:n, 4 * d:].contiguous().view(torch.float64).view(n)

ref = D.QuantisedRefresh(plan, d, 8, cache=Cache, write=write, read=read)
my_mem, my_lu = torch.from_numpy(mem[rank].copy()), torch.from_numpy(lu[rank].copy())
for q in range(Q):
    ref.run(q, my_mem, my_lu)
    mem, lu = orf.boundary_refresh(mem, lu, sets[q], owner)
    assert np.array_equal(my_mem.numpy(), mem[rank]) and np.array_equal(my_lu.numpy(), lu[rank]), q
assert ref.rows_received == sum(len(sets[q][rank]) for q in range(Q)) and ref.rows_sent > 0
dist.barrier()
print("ok", rank)
""" % ROOT


def test_two_ranks_refresh_in_records():
    sock = socket.socket()
    sock.bind(("127.0.0.1", 0))
    port = sock.getsockname()[1]
    sock.close()
    procs = []
    for r in range(2):
        env = dict(os.environ, RANK=str(r), PORT=str(port))
        procs.append(subprocess.Popen([sys.executable, "-c", CODE], env=env, stdout=subprocess.PIPE, stderr=subprocess.PIPE))
    for p in procs:
        out, err = p.communicate(timeout=180)
        assert p.returncode == 0, err.decode()[-3000:]
        assert b"ok" in out
