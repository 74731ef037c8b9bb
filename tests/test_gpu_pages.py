"""GPU: nt_op_kv_resize against a plain simulation, nt_op_kv_keep against plain moves."""
import numpy as np
import pytest

from tests.paged_util import Pages

pytestmark = pytest.mark.gpu


class Plain:
    """The pages of growing and shrinking sequences, by the definition, on the host."""

    def __init__(self, n, page, n_pages, max_pages, seed=0, head=0):
        rng = np.random.default_rng(seed)
        self.page, self.n_pages, self.max_pages = page, n_pages, max_pages
        self.table = np.full((n, max_pages), -1, np.int32)
        self.lens = np.zeros(n, np.int32)
        self.ring = np.roll(rng.permutation(n_pages).astype(np.int32), head)
        self.state = np.array([head, n_pages, 0, 0], np.int32)

    def resize(self, add, max_rows):
        """Does it and returns (off, pos, slot)."""
        n = len(self.lens)
        off, pos, slot = np.zeros(n + 1, np.int32), np.full(max_rows, -1, np.int32), np.full(max_rows, -1, np.int64)
        pages = lambda x: -(-x // self.page)   # noqa: E731
        lens = [int(x) for x in self.lens]
        new = [max(0, x + int(a)) for x, a in zip(lens, add)]
        rows = [max(0, int(a)) for a in add]
        take = sum(max(0, pages(b) - pages(a)) for a, b in zip(lens, new))
        status = max(0, take - int(self.state[1]))
        if sum(rows) > max_rows:
            status = -2
        if max([pages(max(a, b)) for a, b in zip(lens, new)] + [0]) > self.max_pages:
            status = -1
        self.state[2], self.state[3] = status, 0 if status else sum(rows)
        if status:
            return off, pos, slot
        head, count = int(self.state[0]), int(self.state[1])
        tail = head + count
        for b in range(n):
            for p in range(pages(lens[b]), pages(new[b])):
                self.table[b, p] = self.ring[head % self.n_pages]
                head, count = head + 1, count - 1
        for b in range(n):
            for p in range(pages(new[b]), pages(lens[b])):
                self.ring[tail % self.n_pages] = self.table[b, p]
                self.table[b, p] = -1
                tail, count = tail + 1, count + 1
        at = 0
        for b in range(n):
            off[b] = at
            for i in range(rows[b]):
                q = lens[b] + i
                pos[at], slot[at] = q, int(self.table[b, q // self.page]) * self.page + q % self.page
                at += 1
            self.lens[b] = new[b]
        off[n] = at
        self.state[:2] = head % self.n_pages, count
        return off, pos, slot


class Device:
    def __init__(self, plain):
        import torch
        self.p = plain
        for name in ("table", "lens", "ring", "state"):
            setattr(self, name, torch.from_numpy(getattr(plain, name).copy()).cuda())

    def resize(self, add, max_rows, outputs=("off", "pos", "slot"), stream=None, d_add=None):
        import torch
        from paper_2109_08008_amd import nt
        n = len(self.p.lens)
        off = torch.full((n + 1,), 77, dtype=torch.int32, device="cuda")
        pos = torch.full((max(1, max_rows),), 77, dtype=torch.int32, device="cuda")
        slot = torch.full((max(1, max_rows),), 77, dtype=torch.int64, device="cuda")
        if d_add is None:
            d_add = torch.tensor(np.asarray(add, np.int32), device="cuda")
        ptr = lambda name, x: x.data_ptr() if name in outputs else None   # noqa: E731
        nt.nt_op_kv_resize(self.p.page, self.p.n_pages, self.p.max_pages, self.table.data_ptr(), self.lens.data_ptr(),
                           d_add.data_ptr(), n, self.ring.data_ptr(), self.state.data_ptr(), ptr("off", off),
                           ptr("pos", pos), ptr("slot", slot), max_rows, stream)
        torch.cuda.synchronize()
        return off.cpu().numpy(), pos.cpu().numpy()[:max_rows], slot.cpu().numpy()[:max_rows]

    def check(self, what=""):
        held = int(self.p.state[1])
        head = int(self.p.state[0])
        assert self.state.cpu().tolist() == self.p.state.tolist(), what
        assert np.array_equal(self.lens.cpu().numpy(), self.p.lens), what
        assert np.array_equal(self.table.cpu().numpy(), self.p.table), what
        live = (head + np.arange(held)) % self.p.n_pages
        assert np.array_equal(self.ring.cpu().numpy()[live], self.p.ring[live]), what


def step(plain, device, add, max_rows, what=""):
    want = plain.resize(add, max_rows)
    got = device.resize(add, max_rows)
    for g, w, name in zip(got, want, ("off", "pos", "slot")):
        assert np.array_equal(g, w), (what, name)
    device.check(what)


@pytest.mark.parametrize("page", [16, 32, 256])
@pytest.mark.parametrize("n,longest,big", [(1, 1, 3000), (7, 1, 60), (64, 4, 200), (1025, 1, 40), (2100, 3, 9)])
def test_a_life_of_requests(n, longest, big, page):
    """Prompts, steps, rejected tokens, requests that end and new ones in their place."""
    rng = np.random.default_rng(n + page)
    max_pages = -(-(big + 60) // page)
    plain = Plain(n, page, n * max_pages + 1, max_pages, seed=page, head=n % 5)
    device = Device(plain)
    step(plain, device, rng.integers(0, big + 1, n), n * big, "prompts")
    for turn in range(4):
        step(plain, device, rng.integers(0, longest + 1, n), n * longest + 9, "step")
        step(plain, device, -rng.integers(0, longest + 1, n), 0, "rejected")
        mixed = rng.integers(-longest, longest + 1, n)
        mixed[rng.integers(0, n, 1 + n // 8)] = -(2 ** 31)          # requests end
        step(plain, device, mixed, n * longest, "mixed")
        fresh = np.where(plain.lens == 0, rng.integers(0, big // 2 + 1, n), 0)
        step(plain, device, fresh, int(fresh.sum()), "new requests")


def test_all_or_nothing():
    plain = Plain(5, 16, 12, 4, seed=1, head=9)
    device = Device(plain)
    step(plain, device, [30, 0, 17, 16, 1], 64)                     # 6 pages of 12
    step(plain, device, [1, 64, 1, 33, 1], 200, "three pages short")
    assert int(device.state[2]) == 3 - 2                            # needs 0 + 4 + 0 + 3 + 0 = 7 of 6
    step(plain, device, [0, 65, 0, 0, 0], 200, "past the table's row")
    assert int(device.state[2]) == -1
    step(plain, device, [2 ** 31 - 1, 0, 0, 0, 0], 200, "past 2^31")
    assert int(device.state[2]) == -1
    step(plain, device, [1, 1, 1, 1, 1], 4, "more rows than there is room for")
    assert int(device.state[2]) == -2
    step(plain, device, [1, 1, 1, 1, 1], 5)
    assert int(device.state[2]) == 0
    step(plain, device, [-40, 60, -40, 0, 0], 60, "what is given up now is taken later")
    step(plain, device, [30, -60, 0, 0, 40], 70)


@pytest.mark.parametrize("n", [5, 1500])
def test_more_pages_given_up_than_the_ring_has_room_for(n):
    """Lengths and ring that do not match: nothing is done.  With the room, to the page, it is."""
    import torch
    for count, fits in ((100 * n, False), (100 * n - n // 5 + 1, False), (100 * n - n // 5, True)):
        plain = Plain(n, 16, 100 * n, 4, seed=1, head=9)
        plain.lens[:] = np.where(np.arange(n) % 5 == 2, 17, 16)
        plain.table[:, :2] = np.arange(2 * n).reshape(n, 2)
        plain.state[1] = count
        device = Device(plain)
        add = np.where(np.arange(n) % 5 == 2, -1, 0)           # every fifth sequence gives a page up
        add[0] = 0
        if fits:
            step(plain, device, add, 7)
            assert device.state.tolist() == [9, 100 * n, 0, 0]
            continue
        before = [x.clone() for x in (device.table, device.lens, device.ring)]
        off, pos, slot = device.resize(add, 7)
        assert device.state.tolist() == [9, count, -1, 0]
        assert all(torch.equal(a, b) for a, b in zip(before, (device.table, device.lens, device.ring)))
        assert not off.any() and (pos == -1).all() and (slot == -1).all()


@pytest.mark.parametrize("outputs", [(), ("off",), ("pos",), ("slot",)])
def test_outputs_are_optional(outputs):
    for n in (3, 1500):
        plain = Plain(n, 16, 40 * n, 8, seed=2)
        device = Device(plain)
        add = np.arange(n) % 40
        want = plain.resize(add, 40 * n)
        got = device.resize(add, 40 * n if outputs and outputs != ("off",) else 0, outputs)
        device.check()
        for g, w, name in zip(got, want, ("off", "pos", "slot")):
            assert np.array_equal(g, w[:len(g)]) if name in outputs else bool((g == 77).all())


def test_no_sequences():
    import torch
    from paper_2109_08008_amd import nt
    state = torch.tensor([1, 2, 9, 9], dtype=torch.int32, device="cuda")
    x = torch.full((8,), 5, dtype=torch.int32, device="cuda")
    off = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    nt.nt_op_kv_resize(16, 8, 1, x.data_ptr(), x.data_ptr(), x.data_ptr(), 0, x.data_ptr(), state.data_ptr(), off.data_ptr())
    torch.cuda.synchronize()
    assert state.tolist() == [1, 2, 0, 0] and off.tolist() == [0] and x.tolist() == [5] * 8


def test_one_long_prompt_among_many():
    plain = Plain(300, 16, 40000, 20000, seed=3)
    device = Device(plain)
    add = np.ones(300, np.int64)
    add[123] = 200000
    step(plain, device, add, 200400)
    step(plain, device, -add, 0)


def test_rows_up_to_two_to_the_31():
    """As many new rows as a call can have, less 2^16: their numbers stay below 2^31."""
    import torch
    from paper_2109_08008_amd import nt
    n, each, page = 65536, 32767, 256
    per = 128
    i32 = dict(dtype=torch.int32, device="cuda")
    table, ring = torch.full((n, per), -1, **i32), torch.arange(n * per, **i32)
    lens, add, state = torch.zeros(n, **i32), torch.full((n,), each, **i32), torch.tensor([0, n * per, 9, 9], **i32)
    off = torch.empty(n + 1, **i32)
    rows = 2 ** 31 - 1
    guard = torch.full((rows + 4096,), 77, **i32)
    pos = guard[2048:2048 + rows]
    nt.nt_op_kv_resize(page, n * per, per, table.data_ptr(), lens.data_ptr(), add.data_ptr(), n, ring.data_ptr(),
                       state.data_ptr(), off.data_ptr(), pos.data_ptr(), None, rows)
    torch.cuda.synchronize()
    assert state.tolist() == [0, 0, 0, n * each]
    assert bool((lens == each).all()) and bool((off == torch.arange(n + 1, **i32) * each).all())
    assert bool((table.view(-1) == ring).all())
    want = torch.arange(each, **i32)
    for b in range(0, n, 4096):                                # 4096 sequences at a time
        assert bool((pos[b * each:(b + 4096) * each].view(4096, each) == want).all()), b
    assert bool((pos[n * each:] == -1).all())
    assert bool((guard[:2048] == 77).all()) and bool((guard[2048 + rows:] == 77).all())


def test_resize_in_a_graph():
    """A step's growth and the return of a part of it, captured and replayed; counts change between."""
    import torch
    plain = Plain(40, 16, 400, 9, seed=4)
    device = Device(plain)
    step(plain, device, np.arange(40), 1000)
    add, back = (torch.zeros(40, dtype=torch.int32, device="cuda") for _ in range(2))
    from paper_2109_08008_amd import nt
    pos = torch.empty(200, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()

    def call(x, rows):
        nt.nt_op_kv_resize(16, 400, 9, device.table.data_ptr(), device.lens.data_ptr(), x.data_ptr(), 40,
                           device.ring.data_ptr(), device.state.data_ptr(), None, pos.data_ptr() if rows else None, None,
                           rows, torch.cuda.current_stream().cuda_stream)
    with torch.cuda.graph(graph):
        call(add, 200)
        call(back, 0)
    for turn in range(4):
        a, b = np.arange(40) % (turn + 2), -(np.arange(40) % 2)
        add.copy_(torch.from_numpy(a.astype(np.int32)))
        back.copy_(torch.from_numpy(b.astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        _, want, _ = plain.resize(a, 200)
        plain.resize(b, 0)
        device.check(turn)
        assert np.array_equal(pos.cpu().numpy(), want)


# ---- keep ------------------------------------------------------------------------------
def keep(pages, off, path, n_path, stream=None):
    import torch
    from paper_2109_08008_amd import nt
    n = len(off) - 1
    d_off, d_path, d_n = (torch.tensor(np.asarray(x, np.int32), device="cuda") for x in (off, path, n_path))
    add = torch.full((n,), 77, dtype=torch.int32, device="cuda")
    nt.nt_op_kv_keep(pages.cache, d_off.data_ptr(), pages.lens.data_ptr(), d_path.data_ptr(), d_path.shape[1],
                     d_n.data_ptr(), n, add.data_ptr(), stream)
    torch.cuda.synchronize()
    return add.tolist()


def plain_keep(pages, off, path, n_path):
    """(k, v, add) on the host; cells are compared as bits."""
    import torch
    bits = torch.uint8 if pages.fp8 else {"f32": torch.int32, "f16": torch.int16, "bf16": torch.int16}[pages.dtype]
    k, v = (x.cpu().clone().view(bits) for x in (pages.k, pages.v))
    add = []
    for b in range(len(off) - 1):
        new = max(0, off[b + 1] - off[b])
        n = min(max(n_path[b], 0), len(path[b]), new)
        add.append(n - new)
        base = pages.lens_list[b] - new

        def at(p):
            if p < 0 or p // pages.page >= pages.max_pages:
                return None
            pid = int(pages.table_np[b, p // pages.page])
            return (pid, p % pages.page) if 0 <= pid < pages.n_pages else None
        for i in range(n):
            src = path[b][i]
            if src <= i or src >= new:
                continue
            s, d = at(base + src), at(base + i)
            if s and d:
                for x in (k, v):
                    x[d[0], :, d[1]] = x[s[0], :, s[1]].clone()
    return k, v, add


def compare_keep(pages, off, path, n_path):
    import torch
    k, v, add = plain_keep(pages, off, path, n_path)
    got = keep(pages, off, path, n_path)
    assert got == add
    assert torch.equal(pages.k.cpu().view(k.dtype), k) and torch.equal(pages.v.cpu().view(v.dtype), v)


@pytest.mark.parametrize("dtype,fp8", [("f16", False), ("f16", True), ("bf16", False), ("f32", False)])
@pytest.mark.parametrize("kv_heads,d_head", [(1, 32), (3, 64), (8, 128)])
@pytest.mark.parametrize("page", [16, 64])
def test_accepted_branches(page, kv_heads, d_head, dtype, fp8):
    rng = np.random.default_rng(page + d_head)
    new = [0, 1, 5, 24, 64, 16, 30]
    lens = [n + c for n, c in zip(new, (10, 0, 0, 131, 60, 16, 17))]
    pages = Pages(lens, kv_heads, d_head, page, dtype, fp8, seed=page).fill(3)
    off = np.concatenate([[0], np.cumsum(new)]).tolist()
    path = np.full((len(new), 40), -1)
    n_path = []
    for b, n in enumerate(new):
        m = int(rng.integers(0, min(n, 40) + 1))
        path[b, :m] = np.sort(rng.choice(n, m, replace=False)) if m else []
        n_path.append(m)
    path[4, :40], n_path[4] = np.arange(20, 60), 40          # every source is a later destination's neighbour
    compare_keep(pages, off, path.tolist(), n_path)


def test_paths_that_are_none():
    """Empty, too long, out of range and falling paths, holes and positions without a page."""
    new, lens = [6, 6, 6, 6, 6], [20, 40, 6, 30, 3]
    pages = Pages(lens, 2, 64, 16, "f16", seed=1).fill(2)
    table = pages.table_np.copy()
    table[1, 2] = -1
    table[3, 1] = pages.n_pages
    pages.retable(table)
    path = [[5, 3, 4, 9, -2], [1, 3, 5, 0, 0], [0, 1, 2, 3, 4], [2, 3, 4, 5, 0], [1, 2, 3, 4, 5]]
    compare_keep(pages, [0, 6, 12, 18, 24, 30], path, [5, 3, -4, 4, 5])
    pages = Pages(lens, 2, 64, 16, "f16", seed=1).fill(2)
    compare_keep(pages, [0, 6, 12, 18, 24, 30], [[3]] * 5, [2 ** 31 - 1] * 5)
    compare_keep(pages, [0, 6, 12, 10, 24, 30], [[3]] * 5, [1] * 5)


def test_more_new_tokens_than_positions():
    """A context that begins far below position 0: its new tokens there have no page, nothing before the
    table is read, and those from position 0 on move."""
    new, lens = [3000, 2500], [700, 40]
    pages = Pages(lens, 1, 32, 16, "f16", seed=5).fill(6)
    path = [list(range(1, 1500)) + list(range(2301, 2800, 3)), list(range(5, 2000))]
    width = max(len(p) for p in path)
    n_path = [len(p) for p in path]
    compare_keep(pages, [0, 3000, 5500], [p + [-1] * (width - len(p)) for p in path], n_path)
    late = list(range(2400)) + [2450, 2700, 2701, 2999]
    pages = Pages(lens, 1, 32, 16, "f16", seed=5).fill(6)
    compare_keep(pages, [0, 3000, 5500], [late, late], [len(late), 2402])
