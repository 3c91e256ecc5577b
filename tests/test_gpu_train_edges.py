"""The trainer's operators where a call's edges lie: lists cut out of longer ones, launches' limits, what autograd knows."""
import numpy as np
import pytest
import torch

from paper_2210_07768_amd import binding as B
from paper_2210_07768_amd import train as T

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def _lists(rng, n, most, distinct):
    """Values and offsets of a slot whose records have 0 .. most signs each."""
    offsets = np.concatenate([[0], np.cumsum(rng.integers(0, most + 1, n))]).astype(np.int64)
    pool = rng.integers(-(1 << 63), 1 << 63, size=distinct, dtype=np.int64)
    return torch.from_numpy(pool[rng.integers(0, distinct, int(offsets[-1]))]).cuda(), torch.from_numpy(offsets).cuda()


# ------------------------------------------------------------------ lists that leave values out
@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n, most, rows", [(250, 8, 256), (250, 8, 1), (250, 8, 300), (20_000, 6, 4096), (20_000, 6, 5000), (20_000, 40, 1 << 18), (20_000, 40, 200_003),
                                           (300, 3000, 70_001)])
def test_gradient_of_a_window_of_records(n, most, rows, dtype, mean):
    """Records a to b - 1 of longer slots, with room behind the last value: what the records' own signs alone give.  Sums of
    whole numbers are exact.  Of means, terms and their places among the others are the same but for the last row's, whose
    sum may be formed in another order: off by 2^-24 for each of its terms either way, and by the stored result's rounding."""
    rng = np.random.default_rng(n + most + rows)
    slots = [_lists(rng, n, most, 4000) for _ in range(2)]
    one = torch.from_numpy(rng.integers(-(1 << 63), 1 << 63, size=n, dtype=np.int64)).cuda()
    room = torch.from_numpy(rng.integers(-(1 << 63), 1 << 63, size=777, dtype=np.int64)).cuda()
    longer = [torch.cat([v, room]) for v, _ in slots]
    # (scratch of this size as a call leaves it: pairs that would all be taken for terms)
    T.embed_backward(torch.ones(n, 3, 8, device="cuda", dtype=dtype), [T.Signs(longer[0], torch.cat([slots[0][1][:-1], slots[0][1][-1:] + 777])), T.Signs(longer[1], slots[1][1]),
                                                                     T.Signs(one)], rows, mean=mean)
    for a, b in ((0, n), (n // 3, n // 2), (n - 5, n), (0, 1), (7, 7)):
        dout = torch.from_numpy(rng.integers(-8, 9, (b - a, 3, 8)).astype(np.float32)).to(dtype).cuda()
        window = [T.Signs(v, o[a:b + 1]) for v, (_, o) in zip(longer, slots)] + [T.Signs(one[a:b])]
        alone = [T.Signs(v[int(o[a]):int(o[b])].clone(), o[a:b + 1] - o[a]) for v, o in slots] + [T.Signs(one[a:b].clone())]
        got, want = T.embed_backward(dout, window, rows, mean=mean), T.embed_backward(dout, alone, rows, mean=mean)
        if mean:
            assert torch.equal(got[:-1], want[:-1])
            terms = sum(s.values.numel() for s in alone)
            half = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
            size = 8.0 * terms   # (at least the sum of the terms' magnitudes)
            assert bool(((got[-1].double() - want[-1].double()).abs() <= 2 * terms * 2.0 ** -24 * size + 2 * half * want[-1].double().abs() + 2.0 ** -24).all())
        else:
            assert torch.equal(got, want)
        assert torch.equal(got, T.embed_backward(dout, window, rows, mean=mean)), "the same inputs give the same bits"
        table = torch.randn(rows, 8, device="cuda").to(dtype).requires_grad_()
        pooled = T.embed(window, table, b - a, mean=mean)
        assert torch.equal(pooled, T.embed(alone, table.detach(), b - a, mean=mean))
        pooled.backward(dout)
        assert torch.equal(table.grad, got)


def test_gradient_of_few_records_with_much_left_out():
    """One record in the middle of three million values, and no record at all."""
    values = torch.arange(3_000_000, device="cuda")
    dout = torch.full((1, 1, 4), 2.0, device="cuda")
    for rows in (64, 1000, 2_000_000):
        offsets = torch.tensor([1_234_567, 1_234_667], device="cuda")
        want = T.embed_backward(dout, [T.Signs(values[1_234_567:1_234_667].clone(), offsets - 1_234_567)], rows)
        assert float(want.sum()) == 800.0
        assert torch.equal(T.embed_backward(dout, [T.Signs(values, offsets)], rows), want)
        assert not T.embed_backward(dout[:0], [T.Signs(values, offsets[:1])], rows).any()


# ------------------------------------------------------------------ what one launch cannot hold
def _rows_of(values, rows):
    """floor(mix64(sign) x rows / 2^64) in torch's signed integers."""
    shr = lambda x, k: (x >> k) & ((1 << (64 - k)) - 1)  # noqa: E731
    x = (values ^ shr(values, 30)) * (0xBF58476D1CE4E5B9 - (1 << 64))
    x = (x ^ shr(x, 27)) * (0x94D049BB133111EB - (1 << 64))
    x = x ^ shr(x, 31)
    return (shr(x, 32) * rows + (((x & 0xFFFFFFFF) * rows) >> 32)) >> 32


def test_more_records_than_a_launch_holds():
    """2^28 records and some more (a launch's lanes are counted in 32 bits), a list slot's among them."""
    n, rows = (1 << 28) + 1000, 30_011
    table = torch.randn(rows, 1, device="cuda").to(torch.bfloat16)
    values = torch.arange(n, device="cuda")
    offsets = torch.arange(n + 1, device="cuda")
    got = T.embed([T.Signs(values), T.Signs(values, offsets)], table, n)
    for r0 in range(0, n, 1 << 25):
        want = table[_rows_of(values[r0:r0 + (1 << 25)], rows)]
        assert torch.equal(got[r0:r0 + (1 << 25), 0], want) and torch.equal(got[r0:r0 + (1 << 25), 1], want)


def test_more_terms_than_a_launch_holds():
    """2^29 signs and some more whose rows take 64 lanes each: every row's sum is how often signs lead to it."""
    n, arity, rows, dim = 65_536, 8193, 300, 129
    values = torch.arange(n * arity, device="cuda")
    count = torch.zeros(rows, dtype=torch.int64, device="cuda")
    for at in range(0, n * arity, 1 << 26):
        count += torch.bincount(_rows_of(values[at:at + (1 << 26)], rows), minlength=rows)
    got = T.embed_backward(torch.ones(n, 1, dim, device="cuda"), [T.Signs(values, None, arity)], rows)
    assert int(count.max()) < 1 << 24 and torch.equal(got, count.float().unsqueeze(1).expand(rows, dim))


# ------------------------------------------------------------------ AdamW
def test_adamw_8_bit_states_of_unlike_rows():
    """A table's rows whose gradients differ by orders of magnitude, most of them not hit in most steps.  No history of gradients
    moves a weight by more than (1 - beta1) / sqrt((1 - beta2) (1 - beta1^2 / beta2)) = 7.3 times lr (Cauchy-Schwarz on the
    two averages; the bias corrections only lower it); twice that leaves room for the states' rounding."""
    rows, dim = 4096, 16
    for sigma in (2.0, 4.0):
        g = torch.Generator(device="cuda").manual_seed(1)
        scale = 7e-3 * torch.exp(sigma * torch.randn(rows, 1, device="cuda", generator=g))
        often = torch.arange(1, rows + 1, device="cuda").float().rsqrt().unsqueeze(1)
        p = torch.zeros(rows, dim, device="cuda")
        opt = T.AdamW([p], lr=1.0, weight_decay=0.0, bits=8, seed=7)
        most = torch.zeros((), device="cuda")
        for _ in range(300):
            grad = torch.randn(rows, dim, device="cuda", generator=g) * scale * (torch.rand(rows, 1, device="cuda", generator=g) < often)
            p.zero_()
            opt.step([grad])
            most = torch.maximum(most, p.abs().max())
        assert float(most) < 2 * 7.3


@pytest.mark.parametrize("n", [1, 31, 33, 5000, 70_001])
def test_adamw_kept_roots_change_nothing_else(n):
    """The same step with and without: only codes 0 of a sqrt(v) above 0 differ, and they are 1."""
    g = torch.Generator(device="cuda").manual_seed(n)
    r = lambda: torch.randn(n, device="cuda", generator=g) * 10.0 ** torch.randint(-8, 1, (n,), device="cuda", generator=g)  # noqa: E731
    grad, p = r(), torch.randn(n, device="cuda", generator=g)
    grad[n // 2:] *= torch.rand(n - n // 2, device="cuda", generator=g) < 0.5
    sides = []
    for keep in (False, True):
        s = [p.clone(), *(torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)), *(torch.zeros(-(-n // 32), dtype=torch.uint8, device="cuda") for _ in range(2))]
        T.adamw([s[0]], [grad], [s[1]], [s[2]], [s[3]], [s[4]], step=1, seed=5, keep_roots=keep)
        sides.append(s)
    (p0, m0, v0, ms0, vs0), (p1, m1, v1, ms1, vs1) = sides
    assert torch.equal(p0, p1) and torch.equal(m0, m1) and torch.equal(ms0, ms1) and torch.equal(vs0, vs1)
    assert torch.equal(v1, torch.where((v0 == 0) & (grad * grad * 0.001 > 0), 1, v0)) and (n < 5000 or bool(((v0 == 0) & (v1 == 1)).any()))


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("wrong", ["strided gradient", "copies of 16-bit weights", "state of another size", "lr"])
def test_adamw_class_steps_all_weights_or_none(wrong, bits):
    """Two lists by type, of which the second is refused: nothing has moved, and the step that follows is the first one."""
    make = lambda: [torch.full((40,), 0.5, device="cuda"), torch.full((6, 6), 0.25, device="cuda").to(torch.bfloat16)]  # noqa: E731
    grads = lambda: [torch.full((40,), 0.1, device="cuda"), torch.arange(36, device="cuda").view(6, 6).to(torch.bfloat16)]  # noqa: E731
    a, b = make(), make()
    opt, fresh = T.AdamW(a, bits=bits), T.AdamW(b, bits=bits)
    g, lr, kept = grads(), None, opt.m[1]
    if wrong == "strided gradient":
        g[1] = g[1].t()
    elif wrong == "copies of 16-bit weights":
        opt.copies = [torch.zeros_like(w, dtype=torch.bfloat16) for w in a]
    elif wrong == "state of another size":
        opt.m[1] = kept[:-1]
    else:
        lr = float("nan")
    with pytest.raises(B.FbxError):
        opt.step(g, lr=lr)
    assert opt.step_count == 0 and all(torch.equal(x, y) for x, y in zip(a, make()))
    assert not any(bool(t.any()) for t in opt.m + opt.v)
    opt.copies, opt.m[1] = None, kept
    opt.step(grads())
    fresh.step(grads())
    assert opt.step_count == 1 and all(torch.equal(x, y) for x, y in zip(a + opt.m + opt.v, b + fresh.m + fresh.v))


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_class_counts_each_weights_own_steps(bits):
    """A weight whose first gradient comes later than the others' moves as if the optimizer were new, also behind a saved and
    loaded state; a state saved without the weights' counts gives all of them the optimizer's."""
    make = lambda: [torch.full((70,), 0.5, device="cuda"), torch.full((50,), 0.25, device="cuda"), torch.ones(5, device="cuda")]  # noqa: E731
    g = torch.Generator(device="cuda").manual_seed(0)
    first = torch.randn(50, device="cuda", generator=g)
    a = make()
    opt = T.AdamW(a, lr=0.1, bits=bits)
    for _ in range(6):
        opt.step([torch.randn(70, device="cuda", generator=g), None, None])
    saved = {k: [t.clone() for t in x] if isinstance(x, list) else x for k, x in opt.state_dict().items()}
    for o in (opt, T.AdamW([w.clone() for w in a], lr=0.1, bits=bits)):
        o.load_state_dict(saved)
        alone = make()[1]
        T.AdamW([alone], lr=0.1, bits=bits).step([first])
        mine = [w.clone() for w in a]
        o.params = mine
        o.step([torch.ones(70, device="cuda"), first, None])
        assert torch.equal(mine[1], alone) and torch.equal(mine[2], a[2]) and o.step_count == 7 and list(o.steps) == [7, 1, 0]
        old = {k: x for k, x in o.state_dict().items() if k != "steps"}
        o.load_state_dict(old)
        assert list(o.steps) == [7, 7, 7]


# ------------------------------------------------------------------ what autograd knows
def test_results_written_into_a_tensor_are_noted():
    """A tensor that autograd saved and that then takes a result is found changed; one with a history of its own is refused."""
    x, w = torch.randn(8, 6, device="cuda"), torch.randn(5, 6, device="cuda")
    signs, table = [T.Signs(torch.arange(8, device="cuda"))], torch.randn(20, 3, device="cuda")
    for shape, call in (((8, 5), lambda out: T.gated(x, w, w, out=out)), ((8, 1, 3), lambda out: T.embed(signs, table, 8, out=out)),
                        ((20, 3), lambda out: T.embed_backward(torch.ones(8, 1, 3, device="cuda"), signs, 20, out=out))):
        room = torch.ones(shape, device="cuda")
        factor = torch.ones(shape, device="cuda", requires_grad=True)
        product = (factor * room).sum()
        assert call(room).data_ptr() == room.data_ptr()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            product.backward()
        with pytest.raises(B.FbxError):
            call(factor)
        with pytest.raises(B.FbxError):
            call(factor * 2)
        with torch.no_grad():
            assert torch.equal(call(factor), room)


def test_signs_that_changed_before_their_gradient_are_refused():
    """The backward pass reads the signs again: after another extraction into their workspace, or any other write to them, it
    would give another batch's gradient."""
    from paper_2210_07768_amd import workloads as W

    w = W.get(1, 600)
    batches = [[torch.from_numpy(np.asarray(t).copy()).cuda() for t in (raw, off.astype(np.int64))] for raw, off in (w.generate(k * 600, 600) for k in range(2))]
    plan = B.Plan(w.spec)
    table = torch.randn(1000, 4, device="cuda", requires_grad=True)
    want = None
    for static in (False, True):
        into = lambda: torch.empty(1 << 24, dtype=torch.uint8, device="cuda") if static else None  # noqa: E731
        if not static:
            _, ws = B.extract_with_retry(plan, *batches[0])
        for again in (False, True):
            room = into()
            result = plan.extract(*batches[0], out_buffer=room)
            pooled = [T.embed(result, table), T.embed([result.slots[i] for i in result.slot_ids], table, 600)]
            if again:
                plan.extract(*batches[1], out_buffer=room)
                for p in pooled:
                    with pytest.raises(B.FbxError, match="written to"):
                        p.sum().backward()
                continue
            if static:
                plan.extract(*batches[1], out_buffer=into())   # (elsewhere)
            for p in pooled:
                table.grad = None
                p.sum().backward()
                want = table.grad if want is None else want
                assert torch.equal(table.grad, want)
    plan.close()
    values, offsets = torch.arange(12, device="cuda"), torch.tensor([0, 3, 3, 9], device="cuda")
    for write in (lambda: values.add_(1), lambda: offsets[1:2].zero_()):
        pooled = T.embed([T.Signs(values[:3]), T.Signs(values, offsets)], table, 3)
        write()
        with pytest.raises(B.FbxError, match="written to"):
            pooled.sum().backward()
    slots = [T.Signs(values[:3])]
    pooled = T.embed(slots, table, 3)
    slots[0] = T.Signs(values[3:6])   # (the list is the caller's)
    table.grad = None
    pooled.sum().backward()
    assert torch.equal(table.grad, T.embed_backward(torch.ones(3, 1, 4, device="cuda"), [T.Signs(values[:3])], 1000))


# ------------------------------------------------------------------ the runtime's errors
def test_errors_that_others_left_stay_theirs():
    """A call succeeds beside an error that something else left with the HIP runtime, and leaves it there to be found."""
    import ctypes

    path = next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line)
    hip = ctypes.CDLL(path)
    x, w, out = torch.randn(40, 8, device="cuda"), torch.randn(6, 8, device="cuda"), torch.zeros(40, 6, device="cuda")
    signs, table, pooled, grad = [T.Signs(torch.arange(40, device="cuda"))], torch.randn(20, 4, device="cuda"), torch.zeros(40, 1, 4, device="cuda"), torch.zeros(20, 4, device="cuda")
    p, m, v, ones = *(torch.zeros(9, device="cuda") for _ in range(3)), torch.ones(9, device="cuda")   # (torch looks for errors when it computes)
    calls = (lambda: T.gated(x, w, w, out=out), lambda: T.embed(signs, table, 40, out=pooled), lambda: T.embed_backward(pooled, signs, 20, out=grad),
             lambda: T.adamw([p], [ones], [m], [v], step=1))
    for call in calls:
        call()
    for call in calls:
        hip.hipGetLastError()
        assert hip.hipSetDevice(12345) == hip.hipPeekAtLastError() == 101   # (no such device)
        call()
        assert hip.hipPeekAtLastError() == 101
        assert hip.hipGetLastError() == 101
    torch.cuda.synchronize()
    assert bool((grad != 0).any()) and bool((p != 0).all())


# ------------------------------------------------------------------ the ways a large gradient goes
@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("dim, pad, rows, distinct", [(16, 0, 70_001, 1 << 20), (16, 0, 200_003, 3000), (5, 3, 300, 1 << 20), (16, 8, 262_144, 1 << 20), (8, 0, 540_000, 1 << 20), (300, 0, 130_003, 3000),
                                                      (33, 7, 600_011, 1 << 20), (16, 0, 2_000_003, 1 << 20), (2, 2, 1, 1 << 20)])
def test_gradient_of_many_terms(dim, pad, rows, distinct, dtype, mean):
    """Some 350,000 terms: digits of eight and of nine bits, tables most of whose rows have terms and tables where few have, in
    every type.  Lists of 0, 1, 2 or 4 signs, so that whole numbers' sums, and those of their halves and quarters, are exact in
    32 bits (below 2^24 quarters each); what is stored is the nearest of its type."""
    n = 90_007
    rng = np.random.default_rng(dim + rows)
    pool = torch.from_numpy(rng.integers(-(1 << 63), 1 << 63, size=distinct, dtype=np.int64)).cuda()
    g = torch.Generator(device="cuda").manual_seed(rows)
    signs = lambda k: pool[(torch.rand(k, device="cuda", generator=g, dtype=torch.float64) ** 3 * distinct).long()]  # noqa: E731
    lens = torch.tensor([0, 1, 2, 4], device="cuda")[torch.randint(0, 4, (2, n), device="cuda", generator=g)]
    offsets = torch.nn.functional.pad(lens.cumsum(1), (1, 0))
    slots = [T.Signs(signs(n)), *(T.Signs(signs(int(o[-1])), o.contiguous()) for o in offsets)]
    assert sum(s.values.numel() for s in slots) > 1 << 18
    dout = torch.randint(-4, 5, (n, 3, dim), device="cuda", generator=g).to(dtype)
    room = torch.full((rows, dim + pad), 7.0, device="cuda", dtype=dtype)
    T.embed_backward(dout, slots, rows, mean=mean, out=room[:, :dim])
    want = torch.zeros(rows, dim, device="cuda", dtype=torch.float64)
    for i, s in enumerate(slots):
        owner = torch.arange(n, device="cuda") if s.offsets is None else torch.repeat_interleave(torch.arange(n, device="cuda"), lens[i - 1])
        share = 1.0 if s.offsets is None or not mean else 1.0 / lens[i - 1][owner].double().unsqueeze(1)
        want.index_add_(0, _rows_of(s.values, rows), dout[:, i].double()[owner] * share)
    assert torch.equal(room[:, :dim], want.float().to(dtype)) and bool((room[:, dim:] == 7.0).all())
