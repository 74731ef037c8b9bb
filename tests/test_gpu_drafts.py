"""GPU: the operators of requests with drafted tokens, run together: pages for the tokens
(nt_op_kv_resize), a prompt attended to as it arrives (nt_op_attn_prompt) and put into the cache
(nt_op_kv_append), a tree of drafted tokens attended to over it (nt_op_attn_tree), the accepted branch
kept (nt_op_kv_keep) and the rest given back; then one token a sequence (nt_op_attn_paged).  Keys and
values are given, so that each attention has a plain reference over the tokens that were accepted."""
import pytest

from tests.rows_util import assert_rows, attention
from tests.test_gpu_tree import trees

pytestmark = pytest.mark.gpu

HKV, GROUP, DH, PAGE = 2, 3, 64, 16
H = HKV * GROUP
W = (H + 2 * HKV) * DH
SCALE = DH ** -0.5


class Requests:
    """Requests with a cache, driven by the operators; what they hold is tracked on the host."""

    def __init__(self, n, n_pages, max_pages, rows, seed, stream=None):
        import torch
        from paper_2109_08008_amd import nt
        self.n, self.max_pages, self.n_pages, self.rows, self.stream = n, max_pages, n_pages, rows, stream
        ints = lambda *shape, v=0: torch.full(shape, v, dtype=torch.int32, device="cuda")   # noqa: E731
        g = torch.Generator().manual_seed(seed)
        self.k, self.v = (torch.full((n_pages, HKV, PAGE, DH), float("nan"), dtype=torch.float16, device="cuda")
                          for _ in range(2))
        self.table, self.lens, self.add, self.off = ints(n, max_pages, v=-1), ints(n), ints(n), ints(n + 1)
        self.ring = torch.randperm(n_pages, generator=g).to(torch.int32).cuda()
        self.state = torch.tensor([n_pages // 2, n_pages, 0, 0], dtype=torch.int32, device="cuda")
        self.pos = ints(rows)
        self.slot = torch.zeros(rows, dtype=torch.int64, device="cuda")
        self.x = torch.zeros(rows, W, dtype=torch.float16, device="cuda")
        self.mask = torch.zeros(rows, dtype=torch.int64, device="cuda")
        self.out = torch.zeros(rows, H * DH, dtype=torch.float16, device="cuda")
        self.path, self.n_path = ints(n, 8), ints(n)
        self.cache = nt.kv_pages("f16", HKV, DH, PAGE, n_pages, max_pages, self.k.data_ptr(), self.v.data_ptr(),
                                 self.table.data_ptr())
        self.cap = max_pages * PAGE
        self.ws = torch.full((max(256, nt.nt_op_attn_tree_workspace(self.cache, H, n, rows, 16, self.cap),
                                  nt.nt_op_attn_tree_workspace(self.cache, H, n, rows, rows, self.cap),
                                  nt.nt_op_attn_paged_workspace(self.cache, H, n, self.cap)),), 0xFF, dtype=torch.uint8,
                             device="cuda")
        self.held = [[] for _ in range(n)]       # (key, value) rows of each sequence, float64

    def _s(self):
        import torch
        return torch.cuda.current_stream().cuda_stream

    def resize(self, rows):
        from paper_2109_08008_amd import nt
        nt.nt_op_kv_resize(PAGE, self.n_pages, self.max_pages, self.table.data_ptr(), self.lens.data_ptr(),
                           self.add.data_ptr(), self.n, self.ring.data_ptr(), self.state.data_ptr(),
                           self.off.data_ptr() if rows else None, self.pos.data_ptr() if rows else None,
                           self.slot.data_ptr() if rows else None, self.rows if rows else 0, self._s())

    def append(self):
        from paper_2109_08008_amd import nt
        base = self.x.data_ptr()
        nt.nt_op_kv_append(self.cache, base + H * DH * 2, base + (H + HKV) * DH * 2, W, self.off.data_ptr(),
                           self.lens.data_ptr(), self.n, self.rows, self._s())

    def prompt(self):
        from paper_2109_08008_amd import nt
        base = self.x.data_ptr()
        nt.nt_op_attn_prompt("f16", base, W, H, base + H * DH * 2, base + (H + HKV) * DH * 2, W, HKV, DH,
                             self.off.data_ptr(), self.n, self.rows, True, SCALE, self.out.data_ptr(), H * DH, self._s())

    def tree(self, masked=True):
        from paper_2109_08008_amd import nt
        nt.nt_op_attn_tree(self.cache, self.x.data_ptr(), W, H, self.off.data_ptr(), self.mask.data_ptr() if masked else None,
                           self.lens.data_ptr(), self.n, self.rows, 16 if masked else self.rows, self.cap, SCALE, self.out.data_ptr(), H * DH,
                           self.ws.data_ptr(), self.ws.numel(), self._s())

    def keep(self):
        from paper_2109_08008_amd import nt
        nt.nt_op_kv_keep(self.cache, self.off.data_ptr(), self.lens.data_ptr(), self.path.data_ptr(), 8,
                         self.n_path.data_ptr(), self.n, self.add.data_ptr(), self._s())

    def single(self, q, out):
        from paper_2109_08008_amd import nt
        nt.nt_op_attn_paged(self.cache, q.data_ptr(), H * DH, H, self.lens.data_ptr(), self.n, self.cap, SCALE,
                            out.data_ptr(), H * DH, self.ws.data_ptr(), self.ws.numel(), self._s())

    # ---- inputs and references ----
    def load(self, new, seed, masks=None):
        """The step's rows and how many each sequence has."""
        import torch
        g = torch.Generator().manual_seed(seed)
        x = torch.full((self.rows, W), float("nan"))
        x[:sum(new)] = torch.randn(sum(new), W, generator=g)
        self.x.copy_(x.half())
        self.add.copy_(torch.tensor(new, dtype=torch.int32))
        self.out.fill_(7.0)
        if masks is not None:
            words = [w for m in masks for w in m]
            self.mask[:len(words)].copy_(torch.tensor(words))

    def check(self, new, masks=None):
        """The step's outputs; returns each sequence's new (key, value) rows."""
        import torch
        x, got, row, rows = self.x.double(), self.out.reshape(-1, H, DH), 0, []
        assert int(self.state[2]) == 0 and int(self.state[3]) == sum(new)
        for b, n in enumerate(new):
            mine = x[row:row + n]
            k, v = (mine[:, at * DH:(at + HKV) * DH].reshape(n, HKV, DH) for at in (H, H + HKV))
            rows.append(list(zip(k, v)))
            if n:
                old = self.held[b]
                kk = torch.cat([torch.stack([a for a, _ in old]), k]) if old else k
                vv = torch.cat([torch.stack([a for _, a in old]), v]) if old else v
                seen = torch.ones(n, len(old) + n, dtype=torch.bool, device="cuda")
                for i in range(n):
                    for j in range(n):
                        seen[i, len(old) + j] = bool(masks[b][i] >> j & 1) if masks is not None else j <= i
                want, bound = attention(mine[:, :H * DH].reshape(n, H, DH), kk, vv, seen, SCALE, "f16")
                assert_rows(got[row:row + n], want, bound, (b, n))
            row += n
        assert bool((got[row:] == 7.0).all())
        assert self.pos[row:].eq(-1).all() and self.slot[row:].eq(-1).all()
        return rows

    def check_cache(self):
        """The table and pools hold what the sequences do, and every page is somebody's or free."""
        table, lens = self.table.cpu(), self.lens.tolist()
        assert lens == [len(x) for x in self.held]
        used = []
        for b, rows in enumerate(self.held):
            pages = [int(p) for p in table[b] if p >= 0]
            assert len(pages) == -(-len(rows) // PAGE)
            used += pages
            for p, (k, v) in enumerate(rows):
                assert (self.k[pages[p // PAGE], :, p % PAGE].double() == k).all()
                assert (self.v[pages[p // PAGE], :, p % PAGE].double() == v).all()
        head, count = int(self.state[0]), int(self.state[1])
        free = [int(self.ring[(head + i) % self.n_pages]) for i in range(count)]
        assert sorted(used + free) == list(range(self.n_pages))


def branch(parents, r):
    """A random branch of a tree: rising token numbers, each the parent of the next."""
    leaf = r.randrange(len(parents)) if parents else -1
    path = []
    while leaf >= 0:
        path.append(leaf)
        leaf = parents[leaf]
    return path[::-1][:8]


def parents_of(masks):
    return [max([j for j in range(i) if m >> j & 1], default=-1) for i, m in enumerate(masks)]


@pytest.mark.parametrize("graph", [False, True])
def test_prompts_drafts_and_accepted_branches(graph):
    import random
    import torch
    r = random.Random(5)
    q = Requests(5, 60, 10, 96, seed=1)
    new = [30, 1, 0, 17, 40]
    q.load(new, 1)
    q.resize(True)
    q.append()
    q.prompt()
    torch.cuda.synchronize()
    for b, rows in enumerate(q.check(new)):
        q.held[b] += rows
    q.check_cache()

    def step():
        q.resize(True)
        q.append()
        q.tree()

    def accept():
        q.keep()
        q.resize(False)

    graphs = []
    if graph:
        for f in (step, accept):
            gr = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(gr):
                f()
            graphs.append(gr)
    for turn in range(5):
        new = [r.randint(0, 12) for _ in range(q.n)]
        masks = trees(new, seed=turn)
        q.load(new, 10 + turn, masks)
        graphs[0].replay() if graph else step()
        torch.cuda.synchronize()
        rows = q.check(new, masks)
        paths = [branch(parents_of(m), r) for m in masks]
        q.path.copy_(torch.tensor([p + [0] * (8 - len(p)) for p in paths], dtype=torch.int32))
        q.n_path.copy_(torch.tensor([len(p) for p in paths], dtype=torch.int32))
        graphs[1].replay() if graph else accept()
        torch.cuda.synchronize()
        for b, p in enumerate(paths):
            q.held[b] += [rows[b][i] for i in p]
        q.check_cache()
        if turn == 2:       # a request ends, and another takes its place with its prompt in one piece
            q.load([0, 0, 23, 0, 0], 77)
            q.add[0] = -len(q.held[0])
            q.held[0] = []
            q.resize(True)
            q.append()
            q.tree(masked=False)
            torch.cuda.synchronize()
            q.held[2] += q.check([0, 0, 23, 0, 0])[2]
            q.check_cache()
    # one token a sequence over what was kept
    x = torch.randn(q.n, H * DH, generator=torch.Generator().manual_seed(3)).half().cuda()
    out = torch.zeros_like(x)
    q.single(x, out)
    torch.cuda.synchronize()
    for b, rows in enumerate(q.held):
        if rows:
            k, v = torch.stack([a for a, _ in rows]), torch.stack([a for _, a in rows])
            seen = torch.ones(1, len(rows), dtype=torch.bool, device="cuda")
            want, bound = attention(x[b].double().reshape(1, H, DH), k, v, seen, SCALE, "f16")
            assert_rows(out[b].reshape(1, H, DH), want, bound, b)
