"""The paged K/V cache on the GPU: new rows against the oracle, one token's attention against the oracle, a verification pass over pages bit for
bit against the same pass over a dense cache, and the calls together.

Tolerances, with u = 2^-24: a rotated value is the rounding (half a step of its type) of two fp32 products with a cosine and a sine that
are off by at most 1.2e-7 (an angle of at most an eighth of a turn rounded to fp32, 4.7e-8, and 1 ulp of the functions): 3e-7 (|x| + |y|).  A
score of d products summed in fp32 is off by at most d u sum |q_i k_i| and its exponent by 2 u |s| more (scale, subtraction); a weight is
then off by that, relatively, and by 2^-16 (two bf16 parts; 2^-22 in fp32), an output by twice that times max |v|, and by half a step of its type."""
import numpy as np
import pytest
import torch

from oracle import paged as oracle
from paper_2608_27514_b200 import binding as B
from paper_2608_27514_b200.step import VerifyStep

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FP8 = torch.float8_e4m3fn
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "f32": (torch.float32, torch.float32), "e4m3": (torch.bfloat16, FP8)}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24, FP8: 2.0 ** -4}


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _rnd(gen, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device=DEV).to(dtype)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Pool:
    """Pages of random values, handed out in random order; heads and rows may be strided."""

    def __init__(self, kind, tokens, Hkv, d, page, seed=0, spare=3, head_major=False, fill=None):
        self.kind, self.page, self.dtype = kind, page, TYPES[kind][0]
        gen = torch.Generator(device=DEV).manual_seed(seed)
        need = [-(-t // page) for t in tokens]
        n_pages, per = sum(need) + spare, max(1, max(need))
        order = torch.randperm(n_pages, generator=gen, device=DEV)
        table = torch.full((len(tokens), per), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(need):
            table[s, :n] = order[at:at + n].cpu().to(torch.int32)
            at += n
        self.table = table.to(DEV)
        shape = (n_pages, Hkv, page, d) if head_major else (n_pages, page, Hkv, d)
        self.scale = {}
        self.pages = {}
        for name in "kv":
            x = _rnd(gen, *shape)
            x = x.transpose(1, 2) if head_major else x
            if kind == "e4m3":
                self.scale[name] = (0.5 + torch.rand(Hkv, generator=gen, device=DEV)) / 64
                x = (x / self.scale[name][:, None]).clamp(-448, 448).to(FP8)
            else:
                self.scale[name] = None
                x = x.to(TYPES[kind][1])
            self.pages[name] = x
        if fill is not None:  # what nobody may use: rows at or past `fill[s]`, and the spare pages
            live = torch.zeros((n_pages, page), dtype=torch.bool)
            for s, n in enumerate(fill):
                for t in range(min(n, tokens[s])):
                    live[int(table[s, t // page]), t % page] = True
            dead = ~live.to(DEV)
            for x in self.pages.values():
                if kind == "e4m3":
                    x.view(torch.uint8)[dead] = 0x7F
                else:
                    x[dead] = float("nan")
        self.cache = B.make_paged_cache(self.pages["k"], self.pages["v"], self.table, self.scale["k"], self.scale["v"])

    def codes(self, name):
        x = self.pages[name]
        return (x.view(torch.uint8) if self.kind == "e4m3" else x).clone()

    def dense(self, name, s, length):
        """fp64 values of one sequence."""
        x = oracle.ordered(_np(self.pages[name]), self.table[s].cpu().numpy(), length)
        return x if self.scale[name] is None else x * _np(self.scale[name])[None, :, None]


# ------------------------------------------------------------------------------------------ append
def _check_rotated(got, ref, size, dtype):
    tol = HALF_STEP[dtype] * (np.abs(ref) + 3e-7 * size) + 3e-7 * size + (2.0 ** -10 if dtype == FP8 else 1e-38)
    assert (np.abs(got - ref) <= tol).all(), np.abs(got - ref).max()


def _pair_size(x, half, interleaved):
    """|x| + |y| over the pair of every dimension."""
    a = np.abs(np.array(x, dtype=np.float64))
    if half and interleaved:
        s = a[..., 0:2 * half:2] + a[..., 1:2 * half:2]
        a[..., 0:2 * half:2], a[..., 1:2 * half:2] = s, s
    elif half:
        s = a[..., :half] + a[..., half:2 * half]
        a[..., :half], a[..., half:2 * half] = s, s
    return a


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("S,n,Hq,Hkv,d,page,rot,start,ragged", [
    (1, 1, 32, 32, 128, 64, 128, [0], False), (3, 1, 28, 4, 128, 16, 128, [5, 77, 15], False), (2, 37, 4, 4, 64, 8, 64, [3, 100], True),
    (4, 70, 8, 1, 128, 32, 32, [0, 31, 32, 33], True), (2, 5, 3, 3, 64, 1024, 16, [1020, 1023], False), (2, 20, 2, 2, 128, 128, 0, [9, 127], True)])
def test_append(kind, interleaved, S, n, Hq, Hkv, d, page, rot, start, ragged):
    gen = torch.Generator(device=DEV).manual_seed(n + d)
    dt, ct = TYPES[kind]
    pool = Pool(kind, [a + n for a in start], Hkv, d, page, seed=3, head_major=page == 32)
    k, v, q = _rnd(gen, S, n, Hkv, d, dtype=dt), _rnd(gen, S, n, Hkv, d, dtype=dt), _rnd(gen, S, n, Hq, d, dtype=dt)
    n_new = [n, 0, 1, n + 5][:S] if ragged else None
    freq = (1e4 ** (-torch.arange(0, rot, 2, device=DEV) / max(rot, 1))).float() if rot else None
    before = {x: pool.codes(x) for x in "kv"}
    q_out, k_out = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.tsd_append_paged_kv(pool.cache, k, v, _i32(start), None if n_new is None else _i32(n_new), inv_freq=freq, interleaved=interleaved, q=q,
                          q_out=q_out, k_out=k_out, status=status)
    torch.cuda.synchronize()
    assert status.item() == 0
    f = [] if freq is None else _np(freq)
    touched = torch.zeros(pool.pages["k"].shape[:2], dtype=torch.bool, device=DEV)
    for s in range(S):
        m = n if n_new is None else min(n_new[s], n)
        pos = start[s] + np.arange(m)
        at = oracle.slots(start[s], m, pool.table[s].cpu().numpy(), page, pool.cache.n_pages)
        pages, rows = [torch.tensor([a[i] for a in at], dtype=torch.long, device=DEV) for i in (0, 1)]
        touched[pages, rows] = True
        for x, name in ((k, "k"), (v, "v")):
            here = _np(x[s, :m])
            ref = oracle.rotate(here, pos, f if name == "k" else [], interleaved)
            size = _pair_size(here, len(f) if name == "k" else 0, interleaved)
            if name == "k":
                _check_rotated(_np(k_out[s, :m]), ref, size, dt)
            if kind == "e4m3":
                sc = _np(pool.scale[name])[None, :, None]
                ref, size = np.clip(ref / sc, -448, 448), size / sc
            got = _np(pool.pages[name].view(torch.uint8)[pages, rows].view(FP8) if kind == "e4m3" else pool.pages[name][pages, rows])
            _check_rotated(got, ref, size, ct)
            if name == "v" and kind != "e4m3":
                assert np.array_equal(got, here)
        here = _np(q[s, :m])
        _check_rotated(_np(q_out[s, :m]), oracle.rotate(here, pos, f, interleaved), _pair_size(here, len(f), interleaved), dt)
        assert bool((q_out[s, m:] == 7).all()) and bool((k_out[s, m:] == 7).all())       # rows that do not count stay
    for x in "kv":                                                                       # and so do all other slots
        assert torch.equal(pool.codes(x)[~touched], before[x][~touched])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("d,rot", [(128, 16), (128, 48), (128, 64), (128, 112), (64, 16), (64, 32), (64, 48), (128, 0)])
def test_dimensions_that_do_not_turn_are_copied(d, rot, kind, interleaved):
    # behind rotary_dim there may be anything: infinities, NaN and zeros of both signs come out as they are, and the dimensions that turn
    # are those of a call without them, bit for bit
    gen = torch.Generator(device=DEV).manual_seed(rot + d)
    dt, n = TYPES[kind][0], 11
    k, v, q = _rnd(gen, 2, n, 2, d, dtype=dt), _rnd(gen, 2, n, 2, d, dtype=dt), _rnd(gen, 2, n, 6, d, dtype=dt)
    freq = (1e4 ** (-torch.arange(0, rot, 2, device=DEV) / max(rot, 1))).float() if rot else None
    odd = torch.tensor([float("inf"), -0.0, -float("inf"), 1.5, float("nan"), -0.0, -2.5, 0.0, -0.0, -1.0], dtype=dt, device=DEV)

    def run(k, q):
        pool = Pool(kind, [n, n], 2, d, 16, seed=1)
        outs = [torch.zeros_like(q), torch.zeros_like(k)]
        B.tsd_append_paged_kv(pool.cache, k, v, inv_freq=freq, interleaved=interleaved, q=q, q_out=outs[0], k_out=outs[1])
        at = pool.table[:, 0].long()
        return outs + [pool.codes("k")[at][:, :n]]

    def same(a, b):
        bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[a.element_size()]
        return bool(((a.view(bits) == b.view(bits)) | ((a != a) & (b != b))).all())

    plain = run(k, q)
    k2, q2 = k.clone(), q.clone()
    for x in (k2, q2):
        x[..., rot:] = odd[torch.randint(0, len(odd), x[..., rot:].shape, generator=gen, device=DEV)]
    got = run(k2, q2)
    for a, b in zip(got, plain):
        assert same(a[..., :rot].contiguous(), b[..., :rot].contiguous())
    assert same(got[0][..., rot:].contiguous(), q2[..., rot:].contiguous()) and same(got[1][..., rot:].contiguous(), k2[..., rot:].contiguous())
    freq = None                                                                         # the pages hold what a call without rotation puts there
    assert same(got[2][..., rot:].contiguous(), run(k2, q2)[2][..., rot:].contiguous())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("S,n,blocks,Hq,Hkv,d,page,rot", [(40, 131, 1, 6, 2, 128, 16, 128), (45, 120, 2, 28, 4, 64, 64, 32), (32, 160, 3, 4, 1, 128, 32, 112),
                                                          (30, 217, 1, 12, 3, 64, 8, 64), (3, 1901, 1, 8, 8, 128, 128, 128)])
def test_append_of_more_rows_than_warps(kind, interleaved, S, n, blocks, Hq, Hkv, d, page, rot):
    # A warp takes several rows, each of a position and a sequence of its own, the next ones under way while it turns one: more rows than twice
    # the warps.  Rows that do not count, sequences without any and blocks that do not exist lie in between, up to 32 sequences and more.
    rng = np.random.default_rng(S + n)
    new = [int(x) for x in rng.integers(n // 2, n + 1, S)]
    new[1::5] = [0] * len(new[1::5])
    new[-1] = n + 9
    start = [int(x) for x in rng.integers(0, 3 * page, S)]
    block = [int(x) for x in rng.integers(0, blocks, S)]
    if blocks > 1:
        block[2::9] = [blocks, -1, 1 << 30, -(1 << 31), blocks][:len(block[2::9])]
    count = [min(m, n) if 0 <= b < blocks else 0 for m, b in zip(new, block)]
    assert S * n > 2 * 2368
    gen = torch.Generator(device=DEV).manual_seed(n)
    dt, ct = TYPES[kind]
    pool = Pool(kind, [a + n for a in start], Hkv, d, page, seed=2)
    k, v, q = [_rnd(gen, S, blocks * n, h, d, dtype=dt) for h in (Hkv, Hkv, Hq)]
    pos = torch.randint(0, 100000, (S, n), generator=gen, device=DEV, dtype=torch.int32)
    freq = (1e4 ** (-torch.arange(0, rot, 2, device=DEV) / rot)).float()
    before = {x: pool.codes(x) for x in "kv"}
    q_out, k_out = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.tsd_append_paged_kv(pool.cache, k, v, _i32(start), _i32(new), pos, freq, interleaved, q, q_out, k_out, _i32(block) if blocks > 1 else None, n, status)
    assert (status.item() != 0) == (blocks > 1)
    f, where, table = _np(freq), pos.cpu().numpy(), pool.table.cpu().numpy()
    touched = torch.zeros(pool.pages["k"].shape[:2], dtype=torch.bool, device=DEV)
    left = {"q": torch.ones(q.shape[:2], dtype=torch.bool, device=DEV), "k": torch.ones(q.shape[:2], dtype=torch.bool, device=DEV)}
    for s, m in enumerate(count):
        if m == 0:
            continue
        rows = slice(block[s] * n, block[s] * n + m)
        at = oracle.slots(start[s], m, table[s], page, pool.cache.n_pages)
        pages, lines = [torch.tensor([a[i] for a in at], dtype=torch.long, device=DEV) for i in (0, 1)]
        touched[pages, lines] = True
        for x, out, name in ((q, q_out, "q"), (k, k_out, "k"), (v, None, "v")):
            here = _np(x[s, rows])
            ref = here if name == "v" else oracle.rotate(here, where[s, :m], f, interleaved)
            size = _pair_size(here, 0 if name == "v" else len(f), interleaved)
            if out is not None:
                _check_rotated(_np(out[s, rows]), ref, size, dt)
                left[name][s, rows] = False
            if name == "q":
                continue
            if kind == "e4m3":
                sc = _np(pool.scale[name])[None, :, None]
                ref, size = np.clip(ref / sc, -448, 448), size / sc
            got = _np(pool.pages[name].view(torch.uint8)[pages, lines].view(FP8) if kind == "e4m3" else pool.pages[name][pages, lines])
            _check_rotated(got, ref, size, ct)
    assert bool((q_out[left["q"]] == 7).all()) and bool((k_out[left["k"]] == 7).all())
    for x in "kv":
        assert torch.equal(pool.codes(x)[~touched], before[x][~touched])


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_and_negative_positions(interleaved):
    # positions whose angle fp32 does not hold, and a frequency that makes the angle pass 2^32 quarters
    pos = [[1 << 20, 999983, 131071], [0x7fffffff, -1, -131071]]
    freq = torch.tensor([1.0, 0.7310586, 1e-4, 12345.678, 0.0, 3.1415927, 1e-30, 0.25], device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(9)
    k = _rnd(gen, 2, 3, 2, 64)
    out = torch.empty_like(k)
    B.tsd_append_paged_kv(None, k, None, positions=_i32(pos), inv_freq=freq, interleaved=interleaved, k_out=out)
    ref = oracle.rotate(_np(k), np.array(pos), _np(freq), interleaved)
    # numpy's own angle is rounded to 53 bits: 2^31 x 12345 x 2^-53 = 3e-3 at the far end, so it is reduced exactly here
    from fractions import Fraction
    import math
    two_pi = Fraction(2 * math.pi) + Fraction(2.4492935982947064e-16)                  # 2 pi to 106 bits
    exact = np.zeros((2, 3, 8))
    for s in range(2):
        for i in range(3):
            for j in range(8):
                a = Fraction(pos[s][i]) * Fraction(float(freq[j]))
                exact[s, i, j] = float(a - two_pi * round(a / two_pi))
    z = np.exp(1j * exact)[:, :, None]
    x = _np(k)
    re, im = (x[..., 0:16:2], x[..., 1:16:2]) if interleaved else (x[..., :8], x[..., 8:16])
    w = (re + 1j * im) * z
    ref = x.copy()
    if interleaved:
        ref[..., 0:16:2], ref[..., 1:16:2] = w.real, w.imag
    else:
        ref[..., :8], ref[..., 8:16] = w.real, w.imag
    # the kernel's angle in turns is rounded to 53 bits twice: 2^-52 of it, in radians 2^-52 x |angle|
    far = np.abs(np.array(pos))[..., None] * np.abs(_np(freq)) * 2.0 ** -52 * 2
    far = np.concatenate([far, far], -1)[..., None, :] if not interleaved else np.repeat(far, 2, -1)[..., None, :]
    size = _pair_size(x, 8, interleaved)
    tol = 2.0 ** -24 * np.abs(ref) + 3e-7 * size
    tol[..., :16] += far * size[..., :16]
    assert (np.abs(_np(out) - ref) <= tol).all()


def test_positions_counted_on_beyond_31_bits():
    # rotated only, so that no slot has to exist: the second row stands at 2^31
    gen = torch.Generator(device=DEV).manual_seed(10)
    k = _rnd(gen, 1, 2, 2, 64)
    freq = 2.0 ** -torch.arange(20, 28, device=DEV).float()
    out = torch.empty_like(k)
    B.tsd_append_paged_kv(None, k, None, _i32([0x7fffffff]), inv_freq=freq, k_out=out)
    ref = oracle.rotate(_np(k), np.array([[0x7fffffff, 0x80000000]]), _np(freq))
    assert (np.abs(_np(out) - ref) <= 2.0 ** -24 * np.abs(ref) + 3e-7 * _pair_size(_np(k), 8, False) + 1e-30).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_the_accepted_block_goes_to_its_pages(kind):
    # the rows of one node of many, unrotated, the same bytes that the hand-over into a dense cache gives; views with other strides
    S, Bn, R, H, d, page = 3, 7, 32, 4, 64, 16
    gen = torch.Generator(device=DEV).manual_seed(1)
    both = _rnd(gen, S, Bn * R, 2 * H, d, dtype=TYPES[kind][0])
    k, v = both[:, :, :H], both[:, :, H:]
    node, start = _i32([6, 0, 3]), [40, 0, 17]
    pool = Pool(kind, [a + R for a in start], H, d, page)
    B.tsd_append_paged_kv(pool.cache, k, v, _i32(start), block=node, n_rows=R)
    dense = [torch.zeros((S, 80, H, d), dtype=k.dtype, device=DEV) for _ in range(2)]
    B.tsd_gather_accepted_kv(node, R, k, v, dense[0], dense[1], _i32(start))
    for s in range(S):
        for i, name in enumerate("kv"):
            assert np.array_equal(pool.dense(name, s, start[s] + R)[start[s]:], _np(dense[i][s, start[s]:start[s] + R]))


def test_rotation_in_place_and_alone():
    gen = torch.Generator(device=DEV).manual_seed(4)
    q, k = _rnd(gen, 2, 9, 4, 128, dtype=torch.bfloat16), _rnd(gen, 2, 9, 2, 128, dtype=torch.bfloat16)
    freq = torch.rand(32, generator=gen, device=DEV)
    pos = torch.randint(0, 5000, (2, 9), generator=gen, device=DEV, dtype=torch.int32)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    B.tsd_append_paged_kv(None, k, None, positions=pos, inv_freq=freq, q=q, q_out=q_out, k_out=k_out)
    B.tsd_append_paged_kv(None, k, None, positions=pos, inv_freq=freq, q=q, q_out=q, k_out=k)
    assert torch.equal(q, q_out) and torch.equal(k, k_out) and not torch.equal(q[:, :, :, :64], q[:, :, :, 64:])


def test_slots_that_do_not_exist():
    # a page outside the pool, one not handed out, slots in front of and behind the table, a block that is none: reported, not written
    gen = torch.Generator(device=DEV).manual_seed(5)
    pool = Pool("bf16", [40, 40, 40, 40], 2, 64, 8)
    pool.table[1, 3], pool.table[1, 4] = -1, 1 << 30
    k, v, q = [_rnd(gen, 4, 2 * 6, h, 64, dtype=torch.bfloat16) for h in (2, 2, 4)]
    q_out = torch.zeros_like(q)
    start, block = [36, 22, -3, 0], [1, 0, 0, 2]
    before = {x: pool.codes(x) for x in "kv"}
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.tsd_append_paged_kv(pool.cache, k, v, _i32(start), q=q, q_out=q_out, block=_i32(block), n_rows=6, status=status)
    assert B.tsd_check_status(status) == B.TSD_ERR_DEVICE_DATA
    changed = torch.zeros(pool.pages["k"].shape[:2], dtype=torch.bool, device=DEV)
    for s in range(3):
        for i, (p, r) in enumerate(oracle.slots(start[s], 6, pool.table[s].cpu().numpy(), 8, pool.cache.n_pages)):
            if p >= 0:
                changed[p, r] = True
                assert torch.equal(pool.pages["k"][p, r], k[s, block[s] * 6 + i]) and torch.equal(pool.pages["v"][p, r], v[s, block[s] * 6 + i])
        assert torch.equal(q_out[s, block[s] * 6:block[s] * 6 + 6], q[s, block[s] * 6:block[s] * 6 + 6])
    assert int(changed.sum()) == 4 + 2 + 3                                              # slots 36-39; 22, 23; 0-2
    assert not q_out[3].any()
    for x in "kv":
        assert torch.equal(pool.codes(x)[~changed], before[x][~changed])
    # a zero scale, infinities and values beyond 448 scales saturate
    pool = Pool("e4m3", [8], 2, 64, 8)
    x = torch.full((1, 1, 2, 64), float("inf"), dtype=torch.bfloat16, device=DEV)
    B.tsd_append_paged_kv(pool.cache, x, -x)
    assert bool((pool.pages["k"].view(torch.uint8)[int(pool.table[0, 0]), 0] == 0x7E).all())
    assert bool((pool.pages["v"].view(torch.uint8)[int(pool.table[0, 0]), 0] == 0xFE).all())


# ------------------------------------------------------------------------------------------- token
def _token(pool, q, lens, sm_scale, workspace=None, out=None, stream=None):
    S, Hq, d = q.shape
    if workspace is None:
        workspace = torch.zeros(B.tsd_paged_attention_workspace_bytes(pool.cache, Hq), dtype=torch.uint8, device=DEV)
    out = torch.full_like(q, 3.0) if out is None else out
    lse = torch.full((S, Hq), 3.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.tsd_paged_attention(pool.cache, q, lens, out, lse, sm_scale, workspace, status, stream)
    return out, lse, status


def _check_token(pool, q, lens, out, lse, sm_scale, only=None):
    bits = 2.0 ** -22 if q.dtype == torch.float32 else 2.0 ** -16
    for s, n in enumerate(lens):
        if only is not None and s not in only:
            continue
        k, v, qs = pool.dense("k", s, n), pool.dense("v", s, n), _np(q[s])
        ref, ref_lse = oracle.token_attention(qs, k, v, sm_scale)
        if n == 0:
            assert not out[s].any() and bool(torch.isneginf(lse[s]).all())
            continue
        group = qs.shape[0] // k.shape[1]
        for h in range(qs.shape[0]):
            g = h // group
            size = abs(sm_scale) * (np.abs(k[:, g]) @ np.abs(qs[h])).max()
            off = (qs.shape[1] + 4) * 2.0 ** -24 * size                                # of a score
            tol = HALF_STEP[q.dtype] * np.abs(ref[h]) + 2 * (off + bits) * np.abs(v[:, g]).max()
            assert (np.abs(_np(out[s, h]) - ref[h]) <= tol).all(), (s, h, np.abs(_np(out[s, h]) - ref[h]).max())
            assert abs(float(lse[s, h]) - ref_lse[h]) <= off + 2.0 ** -22 * (1 + abs(ref_lse[h]))


@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,d,page,lens", [
    (32, 32, 128, 64, [768]), (28, 4, 128, 16, [0, 1, 2, 15, 16, 17, 300]), (4, 4, 64, 8, [7, 8, 9, 63, 64, 65, 0]), (8, 1, 64, 128, [1000, 0, 127]),
    (2, 1, 128, 32, [31, 33, 1]), (16, 1, 128, 64, [500, 3]), (36, 4, 64, 16, [129, 40]), (40, 1, 128, 1024, [1, 1500]), (12, 3, 64, 256, [2000, 255, 257, 0])])
def test_token_attention(kind, Hq, Hkv, d, page, lens):
    # every type over head layouts (groups of 1 to 40) and lengths around chunks and pages; NaN wherever nothing may be read
    gen = torch.Generator(device=DEV).manual_seed(Hq + page)
    pool = Pool(kind, lens, Hkv, d, page, seed=page, head_major=page == 32, fill=lens)
    q = _rnd(gen, len(lens), Hq, d, dtype=pool.dtype) * 2
    out, lse, status = _token(pool, q, _i32(lens), d ** -0.5)
    torch.cuda.synchronize()
    assert status.item() == 0
    _check_token(pool, q, lens, out, lse, d ** -0.5)


@pytest.mark.parametrize("kind,d", [("bf16", 128), ("f32", 64), ("e4m3", 128)])
@pytest.mark.parametrize("S,Hkv,group,longest", [(1, 4, 7, 4096), (3, 4, 2, 520), (2, 16, 1, 700), (5, 12, 1, 260), (1, 1, 20, 1500), (40, 2, 4, 100), (37, 4, 1, 30)])
def test_short_sequences_in_short_and_in_long_tables(kind, d, S, Hkv, group, longest):
    # blocks are dealt to the sequences' heads by what a sequence may have, or, with room for far more, by what it has
    lens = [longest, 0, 1, longest // 2, 17, 33, longest // 3][:S] + [longest - s for s in range(max(S - 7, 0))]
    pool = Pool(kind, lens, Hkv, d, 16, seed=S, fill=lens)
    gen = torch.Generator(device=DEV).manual_seed(S)
    q = _rnd(gen, S, Hkv * group, d, dtype=pool.dtype)
    for columns in (0, 5000):
        if columns:
            table = torch.full((S, columns), -1, dtype=torch.int32, device=DEV)
            table[:, :pool.table.shape[1]] = pool.table
            pool.cache = B.make_paged_cache(pool.pages["k"], pool.pages["v"], table, pool.scale["k"], pool.scale["v"])
        out, lse, status = _token(pool, q, _i32(lens), d ** -0.5)
        assert status.item() == 0
        _check_token(pool, q, lens, out, lse, d ** -0.5, only=set(range(10)))
        again, lse2, _ = _token(pool, q, _i32(lens), d ** -0.5)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3"])
def test_one_long_sequence_is_cut_and_joined(kind):
    # one sequence over all blocks; the largest scores lie in one stretch, so that the others' parts weigh nothing
    lens = [40000 if kind != "f32" else 20011]
    pool = Pool(kind, lens, 2, 128, 64, fill=lens)
    gen = torch.Generator(device=DEV).manual_seed(2)
    q = _rnd(gen, 1, 14, 128, dtype=pool.dtype)
    for scale in (128 ** -0.5, 4.0, -0.3, 0.0):
        out, lse, _ = _token(pool, q, _i32(lens), scale)
        _check_token(pool, q, lens, out, lse, scale)


def test_many_sequences_and_repeats():
    # more sequences than blocks, many of them empty; the same call gives the same bits, in any workspace that has been used before
    rng = np.random.default_rng(0)
    lens = [int(x) for x in rng.integers(0, 90, 333)]
    lens[::7] = [0] * len(lens[::7])
    lens[100] = 5000
    pool = Pool("bf16", lens, 2, 64, 16, fill=lens)
    gen = torch.Generator(device=DEV).manual_seed(3)
    q = _rnd(gen, len(lens), 6, 64, dtype=torch.bfloat16)
    ws = torch.zeros(B.tsd_paged_attention_workspace_bytes(pool.cache, 6), dtype=torch.uint8, device=DEV)
    out, lse, _ = _token(pool, q, _i32(lens), 0.125, ws)
    _check_token(pool, q, lens, out, lse, 0.125)
    small = Pool("bf16", [70, 3], 2, 64, 16)
    for _ in range(3):
        _token(small, q[:2, :, :].contiguous(), _i32([70, 3]), 0.125, ws)
        again, lse2, _ = _token(pool, q, _i32(lens), 0.125, ws)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("S,every,longest", [(31, 2, 40), (32, 32, 900), (33, 1, 20), (64, 64, 700), (385, 3, 60), (2000, 300, 400), (5000, 7, 12)])
def test_few_sequences_among_many_slots(S, every, longest):
    # a batch with slots to spare: most sequences are empty, at both ends and in long runs between the others
    rng = np.random.default_rng(S)
    lens = [int(rng.integers(1, longest + 1)) if s % every == every - 1 else 0 for s in range(S)]
    pool = Pool("bf16", lens, 2, 64, 16, fill=lens)
    gen = torch.Generator(device=DEV).manual_seed(S)
    q = _rnd(gen, S, 4, 64, dtype=torch.bfloat16)
    out, lse, status = _token(pool, q, _i32(lens), 0.125)
    assert status.item() == 0
    empty = torch.tensor([n == 0 for n in lens], device=DEV)
    assert not out[empty].any() and bool(torch.isneginf(lse[empty]).all())
    some = [s for s, n in enumerate(lens) if n]
    _check_token(pool, q, lens, out, lse, 0.125, only=set(some[:60] + some[-5:]))


@pytest.mark.parametrize("kind,Hkv,lens", [("bf16", 2, [9 * 16 + 5, 0, 3, 40]), ("bf16", 1, [5, 0, 0, 1]), ("f32", 3, [70, 9, 0, 130]), ("e4m3", 4, [33, 600, 0, 1])])
def test_blocks_with_fewer_chunks_than_warps(kind, Hkv, lens):
    # a long table (cut on the device) and few keys: most warps have no chunk, and reach the joining of parts long before the others.  A call
    # of other lengths in between leaves another share in a block's shared memory; every call gives the same bits and leaves every ticket at 0.
    pool = Pool(kind, lens, Hkv, 128, 16, fill=lens)
    table = torch.full((len(lens), 6000), -1, dtype=torch.int32, device=DEV)
    table[:, :pool.table.shape[1]] = pool.table
    pool.cache = B.make_paged_cache(pool.pages["k"], pool.pages["v"], table, pool.scale["k"], pool.scale["v"])
    gen = torch.Generator(device=DEV).manual_seed(1)
    q = _rnd(gen, len(lens), 4 * Hkv, 128, dtype=pool.dtype)
    ws = torch.zeros(B.tsd_paged_attention_workspace_bytes(pool.cache, 4 * Hkv), dtype=torch.uint8, device=DEV)
    out, lse, status = _token(pool, q, _i32(lens), 0.09, ws)
    assert status.item() == 0
    _check_token(pool, q, lens, out, lse, 0.09)
    other = [max(n // 2, 1) if n else 0 for n in lens]
    half, half_lse, _ = _token(pool, q, _i32(other), 0.09, ws)
    _check_token(pool, q, other, half, half_lse, 0.09)
    calls = [(_i32(lens), out, lse), (_i32(other), half, half_lse)]
    for i in range(200):
        n, o, l = calls[i % 2]
        again, lse2, _ = _token(pool, q, n, 0.09, ws)
        assert torch.equal(o, again) and torch.equal(l, lse2)
    assert not ws[:148 * 4].any()


@pytest.mark.parametrize("kind,keys", [("bf16", 16), ("f32", 8), ("e4m3", 32)])
def test_items_of_one_chunk_each(kind, keys):
    # the smallest pieces there are, cut on the device: each is the whole of its item, so that no ticket is ever drawn
    lens = [keys, 1, 0, keys - 1, keys, 3, 0, keys]
    pool = Pool(kind, lens, 5, 128, 8, fill=lens)
    table = torch.full((len(lens), 6000), -1, dtype=torch.int32, device=DEV)
    table[:, :pool.table.shape[1]] = pool.table
    pool.cache = B.make_paged_cache(pool.pages["k"], pool.pages["v"], table, pool.scale["k"], pool.scale["v"])
    gen = torch.Generator(device=DEV).manual_seed(1)
    q = _rnd(gen, len(lens), 10, 128, dtype=pool.dtype)
    ws = torch.zeros(B.tsd_paged_attention_workspace_bytes(pool.cache, 10), dtype=torch.uint8, device=DEV)
    out, lse, status = _token(pool, q, _i32(lens), 0.09, ws)
    assert status.item() == 0 and not ws.any()
    _check_token(pool, q, lens, out, lse, 0.09)


@pytest.mark.parametrize("S,Hkv,group,d,n,at", [(64, 32, 1, 128, 1000, 0), (64, 32, 1, 64, 1000, 999), (40, 4, 8, 128, 5000, 2500), (3, 2, 16, 64, 3000, 0)])
@pytest.mark.parametrize("gap", [9.0, 14.0, 17.5, 18.5, 21.0, 30.0])
def test_e4m3_weights_far_below_the_largest(S, Hkv, group, d, n, at, gap):
    # One key `gap` nats above all others, whose value is 0: what the others come to is all there is.  Scores are 0 and gap, as exact as fp32 has
    # them: a weight is off by 8 u gap (scale, its factor log2 e, subtraction) and 2^-21 (exp2), relatively, an output of values
    # >= 0 by twice that and its own rounding; and by the weights' split, 2^-22 and, a f16 ending at 2^-24 and the largest weight of a warp
    # being 2^7 at least, 2^-32 of the largest per key.
    pool = Pool("e4m3", [n] * S, Hkv, d, 64)
    pool.scale["k"].fill_(gap / 256)
    pool.scale["v"].fill_(1.0)
    k, v = pool.pages["k"], pool.pages["v"]
    k.view(torch.uint8).zero_()
    v.view(torch.uint8).bitwise_and_(0x7F).clamp_(max=0x60)
    v[..., 0] = torch.tensor(1.0).to(FP8)
    page = pool.table[:, at // 64].long()
    k[page, at % 64, :, 0] = torch.tensor(256.0).to(FP8)
    v.view(torch.uint8)[page, at % 64] = 0
    q = torch.zeros((S, Hkv * group, d), dtype=torch.bfloat16, device=DEV)
    q[:, :, 0] = 1.0
    out, lse, _ = _token(pool, q, _i32([n] * S), 1.0)
    small = float(np.exp(np.float64(-np.float32(gap / 256) * np.float64(256))))
    total = 1.0 + (n - 1) * small
    off = 8 * 2.0 ** -24 * gap + 2.0 ** -21
    for s in {0, S // 2, S - 1}:
        rows = torch.arange(n, device=DEV)
        values = _np(v[pool.table[s, rows // 64].long(), rows % 64])
        ref = np.repeat(values.sum(0) * small / total, group, 0)
        tol = (2.0 ** -8 + 2 * off) * ref + (2.0 ** -22 + n * 2.0 ** -32) * values.max()
        assert (np.abs(_np(out[s]) - ref) <= tol).all(), (np.abs(_np(out[s]) - ref) / tol).max()
        assert np.abs(_np(lse[s]) - (gap + np.log(total))).max() <= off + 2.0 ** -22 * (1 + gap)


@pytest.mark.parametrize("kind,Hq,Hkv", [("bf16", 8, 8), ("bf16", 20, 1), ("f32", 4, 2)])
def test_scores_of_minus_infinity_weigh_nothing(kind, Hq, Hkv):
    # the first chunks of one sequence, whole stretches of another, all but the last key of a third; every key of the fourth (0 / 0)
    lens, masked = [300, 9000, 200, 50], [range(0, 64), range(1000, 7000), range(0, 199), range(0, 50)]
    pool = Pool(kind, lens, Hkv, 128, 64)
    pages = pool.pages["k"]
    for s, rows in enumerate(masked):
        at = torch.tensor(list(rows), device=DEV)
        pages[pool.table[s, at // 64].long(), at % 64, :, 3] = -float("inf")
    gen = torch.Generator(device=DEV).manual_seed(1)
    q = _rnd(gen, 4, Hq, 128, dtype=pool.dtype)
    q[:, :, 3] = q[:, :, 3].abs() + 0.5
    out, lse, _ = _token(pool, q, _i32(lens), 128 ** -0.5)
    assert bool(torch.isnan(out[3]).all())
    # the same without those keys, one sequence at a time
    for s in range(3):
        live = [t for t in range(lens[s]) if t not in masked[s]]
        rest = Pool(kind, [len(live)], Hkv, 128, 64)
        for x in "kv":
            rows = pool.pages[x][pool.table[s, torch.tensor(live, device=DEV) // 64].long(), torch.tensor(live, device=DEV) % 64]
            to = torch.arange(len(live), device=DEV)
            rest.pages[x][rest.table[0, to // 64].long(), to % 64] = rows
        _check_token(rest, q[s:s + 1], [len(live)], out[s:s + 1], lse[s:s + 1], 128 ** -0.5)


def test_all_empty_none_and_clamped_lengths():
    pool = Pool("bf16", [64, 64, 64], 2, 64, 16)
    gen = torch.Generator(device=DEV).manual_seed(3)
    q = _rnd(gen, 3, 4, 64, dtype=torch.bfloat16)
    out, lse, _ = _token(pool, q, _i32([0, 0, -5]), 0.125)
    assert not out.any() and bool(torch.isneginf(lse).all())
    out, lse, _ = _token(pool, q, None, 0.125)
    _check_token(pool, q, [64] * 3, out, lse, 0.125)
    more, lse2, status = _token(pool, q, _i32([64, 1 << 30, 0x7fffffff]), 0.125)
    assert torch.equal(out, more) and torch.equal(lse, lse2) and status.item() == 0


def test_pages_that_do_not_exist_read_as_zeros():
    lens = [100, 100, 100]
    pool = Pool("bf16", lens, 2, 128, 16)
    pool.table[1, 2], pool.table[2, 6] = -1, pool.cache.n_pages
    gen = torch.Generator(device=DEV).manual_seed(3)
    q = _rnd(gen, 3, 4, 128, dtype=torch.bfloat16)
    out, lse, status = _token(pool, q, _i32(lens), 0.1)
    assert B.tsd_check_status(status) == B.TSD_ERR_DEVICE_DATA
    _check_token(pool, q, lens, out, lse, 0.1)                                          # the oracle reads zeros there, too
    pool.table[2, 6] = 0
    lens = [100, 32, 96]                                                                # what is not needed is not looked at
    out, lse, status = _token(pool, q, _i32(lens), 0.1)
    assert status.item() == 0
    _check_token(pool, q, lens, out, lse, 0.1)


def test_e4m3_codes_are_read_exactly():
    # every finite code as a value, selected one by one: a query that meets one key only, and one column per head
    codes = [c for c in range(256) if c & 0x7F != 0x7F]
    lens = [1] * len(codes)
    pool = Pool("e4m3", lens, 1, 64, 8, fill=lens)
    pool.scale["k"].fill_(1.0)
    pool.scale["v"].fill_(1.0)
    for s, c in enumerate(codes):
        for x in "kv":
            pool.pages[x].view(torch.uint8)[int(pool.table[s, 0]), 0] = c
    q = torch.full((len(codes), 1, 64), 0.0, dtype=torch.bfloat16, device=DEV)
    q[:, 0, 5] = 1.0
    out, lse, _ = _token(pool, q, _i32(lens), 1.0)
    want = torch.tensor(codes, dtype=torch.uint8).view(FP8).double()
    assert torch.equal(out[:, 0].double().cpu(), want[:, None].expand(-1, 64))
    assert (lse[:, 0].double().cpu() - want).abs().max() <= 2.0 ** -22 * 448


def test_views_and_strides():
    # queries out of a joint projection, an output with padded heads, pages whose K and V lie in one tensor
    gen = torch.Generator(device=DEV).manual_seed(8)
    both = _rnd(gen, 12, 16, 4, 128, dtype=torch.bfloat16)
    table = torch.randperm(12, generator=gen, device=DEV).to(torch.int32).view(2, 6)[:, :5]
    cache = B.make_paged_cache(both[:, :, :2], both[:, :, 2:], table)
    q = _rnd(gen, 2, 12, 128, dtype=torch.bfloat16)[:, 2:10]
    out = torch.full((2, 8, 256), 5.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.zeros(B.tsd_paged_attention_workspace_bytes(cache, 8), dtype=torch.uint8, device=DEV)
    B.tsd_paged_attention(cache, q, _i32([80, 41]), out[:, :, :128], None, 0.1, ws)
    for s, n in enumerate([80, 41]):
        rows = both[table[s].long()].flatten(0, 1)[:n]
        ref, _ = oracle.token_attention(_np(q[s]), _np(rows[:, :2]), _np(rows[:, 2:]), 0.1)
        assert np.abs(_np(out[s, :, :128]) - ref).max() <= 2.0 ** -8 * 5 + 1e-3
    assert bool((out[:, :, 128:] == 5).all())


def test_offsets_beyond_32_bits():
    # pools of 4.6 GB each: the pages in use lie behind the 2^32nd byte
    page, H, d, n_pages = 1024, 8, 128, 4500
    pool = [torch.empty((n_pages, page, H, d), dtype=FP8, device=DEV) for _ in range(2)]
    table = _i32([[4499, 4400, 2]])
    cache = B.make_paged_cache(pool[0], pool[1], table)
    gen = torch.Generator(device=DEV).manual_seed(8)
    k, v = [(_rnd(gen, 1, 2500, H, d) * 20).to(torch.bfloat16) for _ in range(2)]
    B.tsd_append_paged_kv(cache, k, v)
    q = _rnd(gen, 1, H, d, dtype=torch.bfloat16) * 0.1
    out, ws = torch.empty_like(q), torch.zeros(B.tsd_paged_attention_workspace_bytes(cache, H), dtype=torch.uint8, device=DEV)
    B.tsd_paged_attention(cache, q, _i32([2500]), out, None, 0.1, ws)
    kd, vd = [_np(x.clamp(-448, 448).to(FP8)[0]) for x in (k, v)]
    ref, _ = oracle.token_attention(_np(q[0]), kd, vd, 0.1)
    assert np.abs(_np(out[0]) - ref).max() <= 2.0 ** -8 * np.abs(ref).max() + 1e-3 * np.abs(vd).max()


def test_captured_calls_follow_their_inputs():
    # append and attention in one graph, replayed while the cache grows token by token, on a stream of its own
    S, H, d, page = 3, 4, 128, 16
    start = [30, 0, 47]
    pool = Pool("bf16", [a + 20 for a in start], H, d, page)
    gen = torch.Generator(device=DEV).manual_seed(8)
    x = {n: torch.zeros((S, 1, H, d), dtype=torch.bfloat16, device=DEV) for n in "kvq"}
    qr, out, lse = torch.zeros_like(x["q"]), torch.zeros((S, H, d), dtype=torch.bfloat16, device=DEV), torch.zeros((S, H), device=DEV)
    slot, lens = _i32(start), _i32([a + 1 for a in start])
    freq = torch.rand(64, generator=gen, device=DEV)
    ws = torch.zeros(B.tsd_paged_attention_workspace_bytes(pool.cache, H), dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def token():
        B.tsd_append_paged_kv(pool.cache, x["k"], x["v"], slot, inv_freq=freq, q=x["q"], q_out=qr, status=status)
        B.tsd_paged_attention(pool.cache, qr[:, 0], lens, out, lse, 0.09, ws, status)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        token()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            token()
        for step in range(20):
            for n in "kvq":
                x[n].copy_(_rnd(gen, S, 1, H, d, dtype=torch.bfloat16))
            graph.replay()
            _check_token(pool, qr[:, 0], [a + 1 + step for a in start], out, lse, 0.09)
            slot += 1
            lens += 1
        stream.synchronize()
    assert status.item() == 0


def test_two_calls_at_once_in_workspaces_of_their_own():
    lens = [[3000, 77], [1234, 2048]]
    pools = [Pool("bf16", n, 4, 128, 64, seed=i) for i, n in enumerate(lens)]
    gen = torch.Generator(device=DEV).manual_seed(8)
    qs = [_rnd(gen, 2, 28, 128, dtype=torch.bfloat16) for _ in pools]
    alone = [_token(p, q, _i32(n), 0.09)[:2] for p, q, n in zip(pools, qs, lens)]
    streams = [torch.cuda.Stream() for _ in pools]
    spaces = [torch.zeros(B.tsd_paged_attention_workspace_bytes(p.cache, 28), dtype=torch.uint8, device=DEV) for p in pools]
    lt = [_i32(n) for n in lens]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(_token(pools[i], qs[i], lt[i], 0.09, spaces[i])[:2])
    torch.cuda.synchronize()
    for i in range(2):
        for out, lse in got[i]:
            assert torch.equal(out, alone[i][0]) and torch.equal(lse, alone[i][1])


# ------------------------------------------------------------------------------------------ verify
@pytest.mark.parametrize("flags", [0, B.TSD_ATTN_FORCE_SIMT])
@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("S,Bn,R,Nc,Hq,Hkv,d,page,lens", [
    (1, 8, 32, 736, 32, 32, 128, 32, None), (3, 5, 32, 300, 28, 4, 128, 16, [300, 0, 17]), (2, 2, 64, 129, 4, 2, 64, 8, [129, 65]),
    (2, 13, 32, 1100, 8, 8, 64, 64, [1100, 1]), (1, 3, 128, 1000, 2, 1, 128, 1024, None), (2, 4, 32, 500, 6, 1, 128, 128, [64, 500]),
    (1, 1, 32, 5056, 4, 4, 128, 64, None), (2, 3, 32, 0, 2, 2, 128, 16, None)])
def test_verify_over_pages_equals_verify_over_a_dense_cache(flags, kind, S, Bn, R, Nc, Hq, Hkv, d, page, lens):
    if kind == "f32" and flags:
        pytest.skip("fp32 takes the CUDA-core kernel anyway")
    dt = TYPES[kind][0]
    used = [Nc] * S if lens is None else lens
    pool = Pool(kind, [max(Nc, 1)] * S, Hkv, d, page, seed=Nc, head_major=page == 32, fill=used)
    for s, n in enumerate(used):                                                       # pages behind the length: not handed out
        pool.table[s, -(-n // page):] = -1
    gen = torch.Generator(device=DEV).manual_seed(5)
    q, kd, vd = _rnd(gen, S, Bn * R, Hq, d, dtype=dt), _rnd(gen, S, Bn * R, Hkv, d, dtype=dt), _rnd(gen, S, Bn * R, Hkv, d, dtype=dt)
    dense = []
    for name in "kv":
        x = torch.zeros((S, max(Nc, 1), Hkv, d), dtype=torch.float64)
        for s, n in enumerate(used):
            x[s, :n] = torch.from_numpy(pool.dense(name, s, n))
        dense.append(x.float().to(dt).to(DEV)[:, :Nc])
    steps = [VerifyStep(S, Bn, R, Nc, Hq, Hkv, d, 64, 1, dt) for _ in range(2)]
    for st in steps:
        st.build_mask(None, None if lens is None else _i32(lens))
        st.out.fill_(9.0)
    a = steps[0].attention_paged(q, pool.cache, kd, vd, d ** -0.5, flags)
    b = steps[1].attention(q, dense[0] if Nc else None, dense[1] if Nc else None, kd, vd, d ** -0.5, flags)
    for st in steps:
        st.check_status()
    assert torch.equal(a, b) and torch.equal(steps[0].attn_lse, steps[1].attn_lse)
    assert bool(torch.isfinite(a.float()).all())


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_verify_over_missing_pages(kind):
    # in a tile of its own, in the middle of a tile and first of the block's items: zeros, and reported
    S, Nc, page = 2, 400, 16
    pool = Pool(kind, [Nc] * S, 2, 128, page)
    pool.table[0, 0], pool.table[1, 9], pool.table[1, 24] = -1, pool.cache.n_pages, -7
    gen = torch.Generator(device=DEV).manual_seed(5)
    q, kd, vd = [_rnd(gen, S, 64, h, 128, dtype=torch.bfloat16) for h in (4, 2, 2)]
    steps = [VerifyStep(S, 2, 32, Nc, 4, 2, 128, 64, 1, torch.bfloat16) for _ in range(2)]
    a = steps[0].attention_paged(q, pool.cache, kd, vd, 0.1)
    dense = [torch.stack([torch.from_numpy(pool.dense(x, s, Nc)) for s in range(S)]).float().bfloat16().to(DEV) for x in "kv"]
    b = steps[1].attention(q, dense[0], dense[1], kd, vd, 0.1)
    assert torch.equal(a, b) and torch.equal(steps[0].attn_lse, steps[1].attn_lse)
    assert B.tsd_check_status(steps[0].status) == B.TSD_ERR_DEVICE_DATA


def test_verify_refusals_on_a_device():
    pool = Pool("bf16", [64], 2, 128, 16)
    step = VerifyStep(1, 1, 32, 64, 4, 2, 128, 64, 1, torch.bfloat16)
    q, kd = [torch.zeros((1, 32, h, 128), dtype=torch.bfloat16, device=DEV) for h in (4, 2)]
    with pytest.raises(B.TsdError):
        step.attention_paged(q, pool.cache, kd, kd, 0.0)                                # the tensor-core kernel wants a positive scale
    step.attention_paged(q, pool.cache, kd, kd, 0.0, B.TSD_ATTN_FORCE_SIMT)
    for bad in ((q[:, :16], kd), (q.float(), kd), (q, kd[:, :, :1]), (q.cpu(), kd), (q, kd.float())):
        with pytest.raises(AssertionError):
            step.attention_paged(bad[0], pool.cache, bad[1], bad[1], 0.1)


def test_refusals_of_the_binding():
    pool = Pool("bf16", [64, 64], 2, 128, 16)
    q = torch.zeros((2, 4, 128), dtype=torch.bfloat16, device=DEV)
    ws = torch.zeros(B.tsd_paged_attention_workspace_bytes(pool.cache, 4), dtype=torch.uint8, device=DEV)
    ok = dict(q=q, kv_lens=_i32([1, 2]), out=torch.empty_like(q), lse=torch.empty((2, 4), device=DEV), workspace=ws)
    B.tsd_paged_attention(pool.cache, **ok)
    for bad in (dict(q=q[:1]), dict(q=q.cpu()), dict(out=q[:, :2]), dict(out=torch.empty_like(q, dtype=torch.float32)), dict(kv_lens=_i32([1])),
                dict(kv_lens=torch.tensor([1, 2], device=DEV)), dict(kv_lens=torch.tensor([1, 2], dtype=torch.int32)),
                dict(lse=torch.empty((2, 3), device=DEV)), dict(lse=torch.empty((2, 4), device=DEV).bfloat16()), dict(q=q[:, :, :64], out=q[:, :, :64])):
        with pytest.raises(AssertionError):
            B.tsd_paged_attention(pool.cache, **dict(ok, **bad))
    with pytest.raises(B.TsdError):
        B.tsd_paged_attention(pool.cache, **dict(ok, workspace=ws[:64]))
    with pytest.raises(B.TsdError):
        B.tsd_paged_attention(pool.cache, **dict(ok, q=q.half()))
    k = torch.zeros((2, 6, 2, 128), dtype=torch.bfloat16, device=DEV)
    for bad in (dict(v=k[:, :5]), dict(v=k.float()), dict(n_rows=4), dict(q=k), dict(q_out=k), dict(q=k, q_out=k[:, :3]), dict(first_slot=_i32([1])),
                dict(n_new=_i32([1, 2, 3])), dict(positions=_i32([1, 2])), dict(inv_freq=torch.zeros(8, dtype=torch.float64, device=DEV)),
                dict(k_out=k[:, :, :1]), dict(v=k.cpu())):
        with pytest.raises(AssertionError):
            B.tsd_append_paged_kv(pool.cache, k, **dict(dict(v=k), **bad))
    with pytest.raises(B.TsdError):
        B.tsd_append_paged_kv(pool.cache, k, None)


def test_status_and_workspace_are_checked():
    # refused before anything is launched: a kernel reports with a 32-bit atomic, and counts on every byte of a workspace or a mask
    pool = Pool("bf16", [64, 64], 2, 128, 16)
    q, k = [torch.zeros((2, 6, h, 128), dtype=torch.bfloat16, device=DEV) for h in (4, 2)]
    ws = torch.zeros(B.tsd_paged_attention_workspace_bytes(pool.cache, 4), dtype=torch.uint8, device=DEV)
    step = VerifyStep(2, 1, 32, 64, 4, 2, 128, 64, 1, torch.bfloat16)
    step.build_mask()
    qv, kv = [torch.zeros((2, 32, h, 128), dtype=torch.bfloat16, device=DEV) for h in (4, 2)]
    out, lse = torch.empty_like(q[:, 0]), torch.empty((2, 4), device=DEV)

    def calls(status=None, workspace=ws, mask=step.mask):
        return (lambda: B.tsd_append_paged_kv(pool.cache, k, k, status=status),
                lambda: B.tsd_paged_attention(pool.cache, q[:, 0], None, out, lse, 0.1, workspace, status),
                lambda: B.tsd_verify_attention_paged(step.layout, mask, qv, pool.cache, kv, kv, step.out, None, 0.1, workspace, 0, status))

    for status in (torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV).view(torch.uint32),
                   torch.zeros(3, dtype=torch.int32, device=DEV), None):
        for call in calls(status):
            call()
    one = torch.zeros(8, dtype=torch.uint8, device=DEV)
    for status in (one[:1], one[1:5], one[:0].view(torch.int32), torch.zeros(1, dtype=torch.int64, device=DEV), torch.zeros(1, device=DEV),
                   torch.zeros(1, dtype=torch.int32)):
        for call in calls(status):
            with pytest.raises(AssertionError):
                call()
    with pytest.raises(AssertionError):
        calls(workspace=ws[:1].expand(len(ws)))[1]()
    with pytest.raises(AssertionError):
        calls(workspace=torch.zeros(2 * len(ws), dtype=torch.uint8, device=DEV)[::2])[1]()
    with pytest.raises(AssertionError):
        calls(mask=step.mask.view(torch.uint8)[:1].expand(step.mask.nbytes))[2]()


def test_arguments_of_an_append_that_do_not_convert():
    # neither a number of rows that 32 bits do not hold nor a truth value that has none reaches the call
    k = torch.zeros((2, 6, 2, 128), dtype=torch.bfloat16, device=DEV)
    out = torch.full_like(k, 7.0)
    for n_rows in ((1 << 32) + 6, (1 << 32) + 3, -6, 1 << 31):
        with pytest.raises(AssertionError):
            B.tsd_append_paged_kv(None, k, None, k_out=out, n_rows=n_rows)
    with pytest.raises(RuntimeError):
        B.tsd_append_paged_kv(None, k, None, k_out=out, interleaved=torch.ones(2, dtype=torch.bool))
    torch.cuda.synchronize()
    assert bool((out == 7).all())


def test_a_captured_verification_follows_lengths_and_table():
    # one graph of a mask and a pass over pages, replayed while sequences grow and their pages change
    S, Bn, R, Hq, Hkv, d, page, Nc = 2, 3, 32, 8, 2, 128, 16, 320
    for kind in ("bf16", "e4m3"):
        pool = Pool(kind, [Nc] * S, Hkv, d, page, seed=7)
        gen = torch.Generator(device=DEV).manual_seed(8)
        q, kd, vd = [_rnd(gen, S, Bn * R, h, d, dtype=torch.bfloat16) for h in (Hq, Hkv, Hkv)]
        steps = [VerifyStep(S, Bn, R, Nc, Hq, Hkv, d, 64, 1, torch.bfloat16) for _ in range(2)]
        lens = _i32([100, 0])

        def layer(st):
            st.build_mask(None, lens)
            return st.attention_paged(q, pool.cache, kd, vd, 0.09)

        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(stream):
            layer(steps[0])
            stream.synchronize()
            with torch.cuda.graph(graph, stream=stream):
                layer(steps[0])
            for n in ([320, 1], [64, 65], [0, 319], [0, 0]):
                lens.copy_(_i32(n))
                pool.table.copy_(pool.table[:, torch.randperm(pool.table.shape[1], generator=gen, device=DEV)])
                steps[0].out.fill_(5.0)
                graph.replay()
                layer(steps[1])
                assert torch.equal(steps[0].out, steps[1].out) and torch.equal(steps[0].attn_lse, steps[1].attn_lse)
                for s in range(S):
                    keys, values = pool.dense("k", s, n[s]), pool.dense("v", s, n[s])
                    kk, vv = np.concatenate([keys, _np(kd[s, :R])]), np.concatenate([values, _np(vd[s, :R])])
                    ref, _ = oracle.token_attention(_np(q[s, 5]), kk, vv, 0.09)
                    # cached values and weights in bf16, half a step each, and the output's own
                    assert np.abs(_np(steps[0].out[s, 5]) - ref).max() <= 3 * 2.0 ** -8 * np.abs(vv).max()
            stream.synchronize()
        for st in steps:
            st.check_status()


def test_graphs_that_share_a_workspace_and_a_stream_of_the_call():
    # graphs of different shapes, replayed in turn on one stream with one workspace; eager calls on a stream that is not the current one
    lens = [[900, 33, 0], [4000]]
    pools = [Pool("bf16", lens[0], 4, 128, 16, seed=1), Pool("e4m3", lens[1], 2, 64, 64, seed=2)]
    gen = torch.Generator(device=DEV).manual_seed(8)
    qs = [_rnd(gen, 3, 28, 128, dtype=torch.bfloat16), _rnd(gen, 1, 40, 64, dtype=torch.bfloat16)]
    ws = torch.zeros(max(B.tsd_paged_attention_workspace_bytes(p.cache, q.shape[1]) for p, q in zip(pools, qs)), dtype=torch.uint8, device=DEV)
    alone = [_token(p, q, _i32(n), 0.09)[:2] for p, q, n in zip(pools, qs, lens)]
    lt, outs, lses = [_i32(n) for n in lens], [torch.empty_like(q) for q in qs], [torch.empty(q.shape[:2], device=DEV) for q in qs]
    graphs, stream = [torch.cuda.CUDAGraph() for _ in pools], torch.cuda.Stream()
    torch.cuda.synchronize()

    def call(i, where=None):
        B.tsd_paged_attention(pools[i].cache, qs[i], lt[i], outs[i], lses[i], 0.09, ws, stream=where)

    for i in range(2):                                                                  # given by its object and by its number
        call(i, (stream, stream.cuda_stream)[i])
    stream.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], alone[i][0]) and torch.equal(lses[i], alone[i][1])
    with torch.cuda.stream(stream):
        for i in range(2):
            with torch.cuda.graph(graphs[i], stream=stream):
                call(i)
        for turn in range(20):
            for i in range(2):
                outs[i].fill_(1.0)
                graphs[i].replay()
                assert torch.equal(outs[i], alone[i][0]) and torch.equal(lses[i], alone[i][1])
    assert not ws[:148 * 4].any()


def test_shared_pages_and_broadcast_queries():
    # sequences that begin alike share pages, a page may stand twice in a table; one query for all sequences has a stride of 0
    pool = Pool("bf16", [200, 200, 200], 2, 128, 16, seed=4)
    pool.table[1, :8], pool.table[2] = pool.table[0, :8], pool.table[0, 3]
    gen = torch.Generator(device=DEV).manual_seed(8)
    q = torch.nn.Parameter(_rnd(gen, 1, 8, 128, dtype=torch.bfloat16))
    lens = [200, 190, 77]
    out, lse, status = _token(pool, q.expand(3, -1, -1), _i32(lens), 0.09, out=torch.empty((3, 8, 128), dtype=torch.bfloat16, device=DEV))
    assert status.item() == 0
    _check_token(pool, q.detach().expand(3, -1, -1), lens, out, lse, 0.09)


@pytest.mark.parametrize("flags", [0, B.TSD_ATTN_FORCE_SIMT])
def test_a_verification_of_one_query_row_for_every_node(flags):
    # rows with a stride of 0, over bf16 pages too: the bits of the same rows laid out
    pool = Pool("bf16", [64], 2, 128, 16)
    gen = torch.Generator(device=DEV).manual_seed(8)
    row, kd = _rnd(gen, 1, 1, 4, 128, dtype=torch.bfloat16), _rnd(gen, 1, 32, 2, 128, dtype=torch.bfloat16)
    step = VerifyStep(1, 1, 32, 64, 4, 2, 128, 64, 1, torch.bfloat16)
    a = step.attention_paged(row.expand(-1, 32, -1, -1), pool.cache, kd, kd, 0.1, flags).clone()
    assert torch.equal(a, step.attention_paged(row.expand(-1, 32, -1, -1).contiguous(), pool.cache, kd, kd, 0.1, flags))
    step.check_status()


# ---------------------------------------------------------------------------------------- together
def test_a_block_from_prompt_to_next_token():
    """Prompts into pages, a tree's rows rotated, verified over the pages, its accepted node appended, and a token on top: every stage
    against the same work on dense tensors."""
    S, Bn, R, Hq, Hkv, d, page = 3, 4, 32, 8, 2, 128, 16
    prompt = [70, 1, 200]
    gen = torch.Generator(device=DEV).manual_seed(6)
    pool = Pool("bf16", [n + R + 1 for n in prompt], Hkv, d, page, fill=[0] * S)
    freq = (1e4 ** (-torch.arange(0, d, 2, device=DEV) / d)).float()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    bf = torch.bfloat16
    k, v = _rnd(gen, S, 200, Hkv, d, dtype=bf), _rnd(gen, S, 200, Hkv, d, dtype=bf)
    B.tsd_append_paged_kv(pool.cache, k, v, n_new=_i32(prompt), inv_freq=freq, status=status)
    q, kd, vd = _rnd(gen, S, Bn * R, Hq, d, dtype=bf), _rnd(gen, S, Bn * R, Hkv, d, dtype=bf), _rnd(gen, S, Bn * R, Hkv, d, dtype=bf)
    pos = (_i32(prompt)[:, None] + torch.arange(R, device=DEV, dtype=torch.int32).repeat(Bn)).contiguous()
    B.tsd_append_paged_kv(None, kd, None, positions=pos, inv_freq=freq, q=q, q_out=q, k_out=kd)
    step = VerifyStep(S, Bn, R, 256, Hq, Hkv, d, 64, 1, bf)
    cache = B.make_paged_cache(pool.pages["k"], pool.pages["v"], torch.nn.functional.pad(pool.table, (0, 16), value=-1))
    step.build_mask(None, _i32(prompt))
    out = step.attention_paged(q, cache, kd, vd, d ** -0.5)
    rot = lambda x, p: torch.from_numpy(oracle.rotate(_np(x), np.asarray(p), _np(freq)))
    for s, n in enumerate(prompt):
        keys, values = rot(k[s, :n], np.arange(n)).numpy(), _np(v[s, :n])
        for b in range(Bn):
            mine = slice(b * R, (b + 1) * R)
            kk, vv = np.concatenate([keys, _np(kd[s, mine])]), np.concatenate([values, _np(vd[s, mine])])
            ref = np.stack([oracle.token_attention(_np(q[s, b * R + r]), kk, vv, d ** -0.5)[0] for r in (0, 31)])
            assert np.abs(_np(out[s, [b * R, b * R + 31]]) - ref).max() <= 2e-2         # K of the prompt rounded to bf16, weights too
    node = _i32([3, 0, 2])
    B.tsd_append_paged_kv(cache, kd, vd, _i32(prompt), block=node, n_rows=R, status=status)
    k1, v1, q1 = [_rnd(gen, S, 1, h, d, dtype=bf) for h in (Hkv, Hkv, Hq)]
    B.tsd_append_paged_kv(cache, k1, v1, _i32([n + R for n in prompt]), inv_freq=freq, q=q1, q_out=q1, status=status)
    lens = [n + R + 1 for n in prompt]
    got, lse, _ = _token(pool, q1[:, 0], _i32(lens), d ** -0.5)
    _check_token(pool, q1[:, 0], lens, got, lse, d ** -0.5)
    for s, n in enumerate(prompt):                                                      # and the pages hold what was appended
        b = int(node[s])
        assert np.array_equal(pool.dense("k", s, lens[s])[n:n + R], _np(kd[s, b * R:(b + 1) * R]))
        assert np.array_equal(pool.dense("v", s, lens[s]), np.concatenate([_np(v[s, :n]), _np(vd[s, b * R:(b + 1) * R]), _np(v1[s])]))
    assert status.item() == 0
    step.check_status()
