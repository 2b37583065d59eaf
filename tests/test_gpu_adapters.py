"""Many adapters on one projection, on the GPU: the batch's tokens by adapter, the adapter terms and their gradients, against the plain
forms in 64 bits (tests/adapters_util.py)."""
import numpy as np
import pytest
import torch

import adapters_util as au

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qb():
    from paper_2407_17029_amd import binding
    return binding


# ---- tokens by adapter ---------------------------------------------------------------------------------------

GROUPS = [  # count, lengths, which, rows behind the last token
    (1, [1], [0], 0), (1, [0], [0], 1), (3, [1, 1, 1], [2, 0, 2], 0), (3, [5, 0, 70, 64], [1, 1, -1, 1], 3), (2, [64, 64], [0, 0], 0),
    (2, [3, 4], [-1, 7], 1), (1, [1000, 1, 63], [0, 0, 0], 0), (700, [1] * 64, [(37 * i) % 700 for i in range(64)], 0),
    (4, [1] * 300, [i % 5 - 1 for i in range(300)], 4), (8192, [1, 2, 3], [8191, 0, 4000], 0),
    (3, [(i * 7) % 200 for i in range(130)], [(i * i) % 4 for i in range(130)], 50), (2, [], [], 5)]


@pytest.mark.parametrize("count,lengths,which,extra", GROUPS)
def test_groups(qb, count, lengths, which, extra):
    starts = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    T = int(starts[-1]) + extra
    want = au.groups(starts, which, count, T)
    got = qb.qblora_adapter_groups(au.dev(starts), au.dev(which), count, T)
    for name, g, w in zip(("first", "order", "tiles"), got, want):
        assert np.array_equal(g.cpu().numpy(), w), name


def test_groups_of_many_requests(qb):
    r = np.random.Generator(np.random.Philox(key=[1, 2]))
    n, count = 8192, 300
    lengths, which = r.integers(0, 6, n), r.integers(-1, count + 1, n)
    starts = np.concatenate([[0], np.cumsum(lengths)])
    T = int(starts[-1]) + 11
    outs = dict(first=torch.full((count + 1,), 99, dtype=torch.int32, device=au.DEV), order=torch.full((T,), 99, dtype=torch.int32, device=au.DEV),
                tiles=torch.full((au.tile_room(count, T), 4), 99, dtype=torch.int32, device=au.DEV))
    got = qb.qblora_adapter_groups(au.dev(starts), au.dev(which), count, T, **outs)
    for g, w in zip(got, au.groups(starts, which, count, T)):
        assert np.array_equal(g.cpu().numpy(), w)


def test_groups_keep_to_their_arrays(qb):
    """Starts that do not ascend, pass T or share tokens: whatever comes out lies inside, and the guards around the arrays stay."""
    count, T = 3, 40
    room = au.tile_room(count, T)
    for starts, which in (([0, 100, 7, -5], [0, 1, 2]), ([-9, 40, 0, 40], [0, 0, 0]), ([0, 40, 0] * 20, ([0, 2] * 30)[:59]),
                          ([2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 0], [1, 1, 1])):
        flat = torch.full((4 * room + count + 1 + T + 64,), 77, dtype=torch.int32, device=au.DEV)
        tiles, first, order = flat[16:16 + 4 * room].view(room, 4), flat[16 + 4 * room:][:count + 1], flat[16 + 4 * room + count + 1:][:T]
        qb.qblora_adapter_groups(au.dev(starts), au.dev(which), count, T, first=first, order=order, tiles=tiles)
        f = flat.cpu().numpy()
        assert (f[:16] == 77).all() and (f[16 + 4 * room + count + 1 + T:] == 77).all()
        o, fi = order.cpu().numpy(), first.cpu().numpy()
        assert ((fi >= 0) & (fi <= T)).all() and ((o >= -1) & (o < T)).all()


# ---- forward and backward ------------------------------------------------------------------------------------

LAYERS = [  # seed, d_in, d_out, lam1, lam2, ranks, lengths, which, rows behind the last token
    (1, 64, 64, 1, 1, [8], [1], [0], 0),
    (2, 64, 128, 2, 2, [16, 8], [1, 1, 1], [1, 0, 1], 2),
    (3, 512, 512, 2, 2, [32], [9], [0], 0),
    (4, 512, 256, 4, 2, [64, 0, 24], [3, 70, 5, 2, 1], [0, 1, 2, -1, 2], 1),
    (5, 256, 576, 8, 8, [40, 16], [17, 33], [1, 0], 0),
    (6, 1024, 640, 2, 4, [128, 64, 128], [64, 65, 1, 128], [0, 2, 1, 0], 0),
    (7, 320, 192, 1, 2, [136], [130], [0], 0),
    (8, 512, 512, 2, 1, [256, 248], [40, 20, 12], [0, 1, 0], 0),
    (9, 256, 256, 2, 2, [512], [20], [0], 0),
    (10, 2048, 1088, 2, 2, [16, 16, 16, 16, 16], [1] * 12, [0, 1, 2, 3, 4, 0, 1, -1, 9, 0, 0, 3], 0),
    (11, 512, 768, 4, 8, [96, 8, 48], [200, 1, 31, 7, 400], [2, 0, 1, 1, 2], 5),
    (12, 192, 320, 8, 1, [512, 264], [16, 8, 9], [1, 0, 1], 0),
    (13, 4096, 2048, 2, 2, [128] * 3, [1, 5, 2, 8, 1], [2, 0, 1, 0, 2], 0),
]


def strided(x, extra=24):
    """The same rows, further apart."""
    out = torch.zeros(x.shape[0], x.shape[1] + extra, dtype=x.dtype, device=x.device)[:, 8:8 + x.shape[1]]
    out.copy_(x)
    return out


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("layer", LAYERS)
def test_forward(qb, layer, apart):
    b = au.Batch(*layer)
    X, Y = (strided(t) if apart else t for t in (au.dev_bf16(b.X), au.dev_bf16(b.Y)))
    out = qb.qblora_adapters_fwd(b.table(qb, R=max(b.ranks) + 8 * apart if max(b.ranks) < 512 else 512), b.groups(qb), X, Y)
    assert out is Y
    want, size = b.forward()
    active = np.array([a >= 0 and b.ranks[a] > 0 for a in b.owner])
    au.assert_rows(Y, want, size, np.where(active, 0, -1), b.Y, b.d_in, max(b.ranks), "Y")
    if apart:                                                # what lies between the rows stays
        assert not Y._base[:, :8].any() and not Y._base[:, 8 + b.d_out:].any()


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("layer", LAYERS)
def test_backward(qb, layer, kept):
    b = au.Batch(*layer)
    grads = b.grads()
    table, groups = b.table(qb, grads=grads), b.groups(qb)
    X, dY, dX = au.dev_bf16(b.X), au.dev_bf16(b.dY), au.dev_bf16(b.dX)
    saved = None
    if kept:
        saved = torch.full((qb.qblora_adapters_saved_bytes(table, b.T),), 255, dtype=torch.uint8, device=au.DEV)
        qb.qblora_adapters_fwd(table, groups, X, au.dev_bf16(b.Y), saved=saved)
    else:
        X, dY, dX = strided(X), strided(dY, 40), strided(dX)
    qb.qblora_adapters_bwd(table, groups, X, dY, dX=dX, saved=saved)
    wX, wA, wB, sX, sA, sB = b.backward()
    active = np.array([a >= 0 and b.ranks[a] > 0 for a in b.owner])
    au.assert_rows(dX, wX, sX, np.where(active, 0, -1), b.dX, b.d_out, max(b.ranks), "dX")
    for a, g in enumerate(grads):
        if g is None:
            continue
        au.assert_grad(g[0], wA[a], sA[a], b.d_out + b.T, f"dA of {a}")
        au.assert_grad(g[1], wB[a], sB[a], b.d_in + b.T, f"dB of {a}")


RULES = [  # inner rank, lambdas, tokens of each adapter: both sides of what chooses a kernel's form
    (256, 2, 2, [1, 2, 3, 4, 5]), (256, 2, 2, [8, 9, 15, 16, 17]), (256, 1, 1, [20, 33, 36, 48, 52]), (264, 2, 2, [1, 4, 5, 17]),
    (128, 4, 4, [4, 5, 21, 36]), (32, 8, 8, [1, 3, 5, 64, 68]), (64, 2, 8, [2, 6, 70]), (24, 2, 1, [3, 63, 65]),
    (16, 2, 2, [1000, 23]), (16, 2, 2, [1000, 24]), (48, 1, 4, [1000, 25, 300])]


@pytest.mark.parametrize("R,lam1,lam2,tokens", RULES)
def test_around_the_rules(qb, R, lam1, lam2, tokens):
    """Forward, and the backward pass without gradients, which takes other forms than the one with them."""
    b = au.Batch(R + len(tokens), 512, 832, lam1, lam2, [R if i % 2 == 0 else max(8, R // 2 // 8 * 8) for i in range(len(tokens))], tokens,
                 list(range(len(tokens))), extra=0)
    table, groups = b.table(qb), b.groups(qb)
    X, Y, dY, dX = (au.dev_bf16(t) for t in (b.X, b.Y, b.dY, b.dX))
    qb.qblora_adapters_fwd(table, groups, X, Y)
    want, size = b.forward()
    au.assert_rows(Y, want, size, b.owner, b.Y, b.d_in, R, "Y")
    qb.qblora_adapters_bwd(table, groups, None, dY, dX=dX, gradients=False)
    want, _, _, size, _, _ = b.backward()
    au.assert_rows(dX, want, size, b.owner, b.dX, b.d_out, R, "dX")


def test_rows_far_apart(qb):
    """Arrays whose rows lie 2^24 elements apart, so that the last ones begin beyond 2^32 elements."""
    b = au.Batch(60, 256, 384, 2, 2, [32, 16], [150, 3, 150], [0, 1, 1])
    far = 1 << 24

    def spread(x):
        out = torch.empty((b.T - 1) * far + x.shape[1], dtype=torch.bfloat16, device=au.DEV).as_strided(x.shape, (far, 1))
        out.copy_(au.dev_bf16(x))
        return out

    grads = b.grads()
    table, groups = b.table(qb, grads=grads), b.groups(qb)
    X, Y, dY, dX = (spread(t) for t in (b.X, b.Y, b.dY, b.dX))
    qb.qblora_adapters_fwd(table, groups, X, Y)
    qb.qblora_adapters_bwd(table, groups, X, dY, dX=dX)
    want, size = b.forward()
    au.assert_rows(Y, want, size, b.owner, b.Y, b.d_in, 32, "Y")
    wX, wA, wB, sX, sA, sB = b.backward()
    au.assert_rows(dX, wX, sX, b.owner, b.dX, b.d_out, 32, "dX")
    for a, g in enumerate(grads):
        au.assert_grad(g[0], wA[a], sA[a], b.d_out + b.T, "dA")
        au.assert_grad(g[1], wB[a], sB[a], b.d_in + b.T, "dB")


def test_backward_of_long_groups(qb):
    """Enough tokens of few adapters that the gradients are summed in slices."""
    b = au.Batch(21, 128, 192, 2, 2, [16, 8, 24], [1500, 700, 1, 1333], [0, 2, 1, 0], 3)
    grads = b.grads()
    table, groups = b.table(qb, grads=grads), b.groups(qb)
    X, dY = au.dev_bf16(b.X), au.dev_bf16(b.dY)
    qb.qblora_adapters_bwd(table, groups, X, dY)
    _, wA, wB, _, sA, sB = b.backward()
    for a, g in enumerate(grads):
        au.assert_grad(g[0], wA[a], sA[a], b.d_out + b.T, f"dA of {a}")
        au.assert_grad(g[1], wB[a], sB[a], b.d_in + b.T, f"dB of {a}")
    again = [tuple(t.clone() for t in g) for g in grads]
    qb.qblora_adapters_bwd(table, groups, X, dY)
    assert all(torch.equal(x, y) for g, h in zip(grads, again) for x, y in zip(g, h))


@pytest.mark.parametrize("dx,gradients", [(True, False), (False, True)])
def test_half_a_backward_pass(qb, dx, gradients):
    """What is not asked for stays, and what is has the bits of the whole pass."""
    b = au.Batch(*LAYERS[5])
    grads = b.grads()
    table, groups = b.table(qb, grads=grads), b.groups(qb)
    X, dY, dX = au.dev_bf16(b.X), au.dev_bf16(b.dY), au.dev_bf16(b.dX)
    full = dX.clone()
    qb.qblora_adapters_bwd(table, groups, X, dY, dX=full)
    want = [tuple(t.clone() for t in g) for g in grads]
    for g in grads:
        for t in g:
            t.fill_(7.0)
    qb.qblora_adapters_bwd(table, groups, X if gradients else None, dY, dX=dX if dx else None, gradients=gradients)
    if dx:
        assert torch.equal(dX, full)
    for g, w in zip(grads, want):
        for t, u in zip(g, w):
            assert torch.equal(t, u) if gradients else (t == 7.0).all()


def test_no_tokens(qb):
    b = au.Batch(30, 128, 128, 2, 2, [16, 8], [0], [0], 0)
    grads = b.grads()
    table, groups = b.table(qb, grads=grads), b.groups(qb)
    none = torch.empty(0, 128, dtype=torch.bfloat16, device=au.DEV)
    assert qb.qblora_adapters_fwd(table, groups, none, none.clone()).shape == (0, 128)
    qb.qblora_adapters_bwd(table, groups, none, none.clone(), dX=none.clone())
    assert all(not t.any() for g in grads for t in g)


def test_some_adapters_without_gradients(qb):
    b = au.Batch(*LAYERS[5])
    grads = b.grads()
    grads[1] = None
    table, groups = b.table(qb, grads=grads), b.groups(qb)
    qb.qblora_adapters_bwd(table, groups, au.dev_bf16(b.X), au.dev_bf16(b.dY))
    _, wA, wB, _, sA, sB = b.backward()
    for a in (0, 2):
        au.assert_grad(grads[a][0], wA[a], sA[a], b.d_out + b.T, "dA")
        au.assert_grad(grads[a][1], wB[a], sB[a], b.d_in + b.T, "dB")


def test_adapters_are_read_when_a_call_runs(qb):
    """An adapter that is stepped in place, and one that another takes the number of."""
    b = au.Batch(*LAYERS[6])
    table, groups = b.table(qb, R=256), b.groups(qb)
    X, Y = au.dev_bf16(b.X), au.dev_bf16(b.Y)
    table.adapters[0].A.copy_(au.dev_bf16(2.0 * b.A[0]))
    qb.qblora_adapters_fwd(table, groups, X, Y)
    b.A[0] = 2.0 * b.A[0]
    want, size = b.forward()
    au.assert_rows(Y, want, size, b.owner, b.Y, b.d_in, 136, "Y")
    c = au.Batch(99, b.d_in, b.d_out, b.lam1, b.lam2, [200], [b.T], [0])
    qb.qblora_adapter_table(c.adapters(qb), b.d_in, b.d_out, into=table, first=0)
    Y = au.dev_bf16(c.Y)
    qb.qblora_adapters_fwd(table, groups, au.dev_bf16(c.X), Y)
    want, size = c.forward()
    au.assert_rows(Y, want, size, c.owner, c.Y, c.d_in, 200, "Y")


def test_infinite_and_nan_rows_stay_theirs(qb):
    """A token whose inputs are not finite spoils its own row and no other of its tile; neither do places behind the tile's last token."""
    b = au.Batch(40, 256, 256, 2, 2, [64, 32], [20, 30, 5], [0, 1, 0], 2)
    b.X[3, 7], b.X[25, 100], b.X[-1, 0] = np.nan, np.inf, np.nan
    X, Y = au.dev_bf16(b.X), au.dev_bf16(b.Y)
    qb.qblora_adapters_fwd(b.table(qb), b.groups(qb), X, Y)
    got = au.host(Y)
    assert np.isnan(got[3]).all() and not np.isfinite(got[25]).any()
    keep = np.ones(b.T, bool)
    keep[[3, 25]] = False
    b.X[~np.isfinite(b.X)] = 0.0
    want, size = b.forward()
    au.assert_rows(au.dev_bf16(got[keep]), want[keep], size[keep], b.owner[keep], b.Y[keep], b.d_in, 64, "Y")


@pytest.mark.parametrize("saved", [False, True])
@pytest.mark.parametrize("tokens", [1, 4, 6, 20, 70])
def test_infinite_sums_pass(qb, tokens, saved):
    """An infinite rank sum, and one next to fp32's largest number, through the parts that the second product takes: what fp32
    products give, no NaN."""
    b = au.Batch(42, 128, 192, 1, 2, [16], [tokens], [0])
    b.A[0], b.B[0], b.s = np.abs(b.A[0]) + 0.25, np.abs(b.B[0]) + 0.25, [1.0]
    b.A[0], b.B[0] = au.bf16(b.A[0]), au.bf16(b.B[0])
    b.X[0, 5] = np.inf
    last = tokens - 1
    if last:
        b.X[last] = 0.0
        b.A[0][7] = 1.0
        b.X[last, 7] = float(torch.finfo(torch.bfloat16).max)
        b.B[0][:, :] = 2.0 ** -6
    table, groups = b.table(qb), b.groups(qb)
    keep = torch.empty(qb.qblora_adapters_saved_bytes(table, b.T), dtype=torch.uint8, device=au.DEV) if saved else None
    Y = au.dev_bf16(b.Y)
    qb.qblora_adapters_fwd(table, groups, au.dev_bf16(b.X), Y, saved=keep)
    got = au.host(Y)
    assert (got[0] == np.inf).all()
    if last:
        want = b.X[last, 7] * 16 * 2.0 ** -6
        assert np.abs(got[last] - want).max() <= want * 2.0 ** -7


def test_workspace_of_a_larger_batch(qb):
    """One workspace, asked for once for the largest batch, full of NaN before every call."""
    b = au.Batch(*LAYERS[10])
    grads = b.grads()
    table = b.table(qb, grads=grads)
    ws = torch.empty(qb.qblora_adapters_workspace_bytes(table, 1500) // 4, device=au.DEV)
    X, dY, dX = au.dev_bf16(b.X), au.dev_bf16(b.dY), au.dev_bf16(b.dX)
    Y, groups = au.dev_bf16(b.Y), b.groups(qb)
    ws.fill_(float("nan"))
    qb.qblora_adapters_fwd(table, groups, X, Y, workspace=ws)
    ws.fill_(float("nan"))
    qb.qblora_adapters_bwd(table, groups, X, dY, dX=dX, workspace=ws)
    want, size = b.forward()
    au.assert_rows(Y, want, size, b.owner, b.Y, b.d_in, 96, "Y")
    wX, wA, wB, sX, sA, sB = b.backward()
    au.assert_rows(dX, wX, sX, b.owner, b.dX, b.d_out, 96, "dX")
    for a, g in enumerate(grads):
        au.assert_grad(g[0], wA[a], sA[a], b.d_out + b.T, "dA")
        au.assert_grad(g[1], wB[a], sB[a], b.d_in + b.T, "dB")


def test_broken_groups_stay_inside(qb):
    """Tiles and token numbers out of range do nothing; rows around the arrays stay."""
    b = au.Batch(41, 128, 128, 2, 2, [16, 8], [70, 5], [0, 1])
    grads = b.grads()
    table = b.table(qb, grads=grads)
    first, order, tiles = (t.clone() for t in b.groups(qb))
    order[::3] = torch.tensor([-1, 2 ** 31 - 1, 1000] * 9, dtype=torch.int32, device=au.DEV)[:len(order[::3])]
    tiles[0] = torch.tensor([0, 60, 64, 0])
    tiles[1] = torch.tensor([-1, 0, 5, 0])
    tiles[2] = torch.tensor([2, 0, 5, 0])
    first[1], first[2] = 2 ** 31 - 1, -5
    room = torch.full((b.T + 128, 128), 3.0, dtype=torch.bfloat16, device=au.DEV)
    Y = room[64:64 + b.T]
    qb.qblora_adapters_fwd(table, (first, order, tiles), au.dev_bf16(b.X), Y)
    qb.qblora_adapters_bwd(table, (first, order, tiles), au.dev_bf16(b.X), au.dev_bf16(b.dY), dX=Y)
    assert (room[:64] == 3.0).all() and (room[64 + b.T:] == 3.0).all()


def test_refusals_of_the_binding(qb):
    b = au.Batch(*LAYERS[1])
    table, groups = b.table(qb), b.groups(qb)
    X, Y = au.dev_bf16(b.X), au.dev_bf16(b.Y)
    for bad in (dict(X=X.float()), dict(Y=Y[:, :64]), dict(X=X[:, ::2]), dict(groups=(groups[0], groups[1][:-1], groups[2])),
                dict(groups=(groups[0], groups[1], groups[2][:-1])), dict(X=X.cpu())):
        args = {**dict(groups=groups, X=X, Y=Y), **bad}
        with pytest.raises(AssertionError):
            qb.qblora_adapters_fwd(table, args["groups"], args["X"], args["Y"])
    with pytest.raises(qb.QBLoRAError):                      # rows that are no multiple of 16 bytes apart
        qb.qblora_adapters_fwd(table, groups, X, strided(Y, 20))
    with pytest.raises(qb.QBLoRAError):
        qb.qblora_adapters_fwd(table, groups, X, Y, workspace=torch.empty(256, dtype=torch.uint8, device=au.DEV))


def test_another_device(qb, monkeypatch):
    """Arrays of a device that is not the current one are refused (here the current one is said to be another)."""
    b = au.Batch(*LAYERS[1])
    table, groups = b.table(qb), b.groups(qb)
    X, Y = au.dev_bf16(b.X), au.dev_bf16(b.Y)
    w = [torch.zeros(5, device=au.DEV)]
    lst = qb.qblora_adamw_list([None], w, w, w, master=w)
    monkeypatch.setattr(qb, "_current_device", lambda: 1)
    for call in (lambda: qb.qblora_adapters_fwd(table, groups, X, Y), lambda: qb.qblora_adapters_bwd(table, groups, X, Y),
                 lambda: b.groups(qb), lambda: b.table(qb), lambda: qb.qblora_adamw_list([None], w, w, w, master=w),
                 lambda: qb.qblora_grad_norm(lst, 1.0), lambda: qb.qblora_adamw_step(lst, 1, 1e-3)):
        with pytest.raises(AssertionError):
            call()


def test_arrays_in_host_memory(qb):
    """Each array that a call takes, in host memory instead: refused before anything is launched."""
    b = au.Batch(*LAYERS[1])
    grads = b.grads()
    table, groups = b.table(qb, grads=grads), b.groups(qb)
    X, Y = au.dev_bf16(b.X), au.dev_bf16(b.Y)
    dY, dX = au.dev_bf16(b.dY), au.dev_bf16(b.dX)
    saved = torch.empty(qb.qblora_adapters_saved_bytes(table, b.T), dtype=torch.uint8, device=au.DEV)
    workspace = torch.empty(qb.qblora_adapters_workspace_bytes(table, b.T), dtype=torch.uint8, device=au.DEV)
    first, order, tiles = groups
    starts, which = au.dev(b.starts), au.dev(b.which)
    calls = [(qb.qblora_adapters_fwd, dict(groups=groups, X=X, Y=Y, saved=saved, workspace=workspace)),
             (qb.qblora_adapters_bwd, dict(groups=groups, X=X, dY=dY, dX=dX, saved=saved, workspace=workspace))]
    for call, arrays in calls:
        for name, value in arrays.items():
            others = [value.cpu()] if name != "groups" else [(first.cpu(), order, tiles), (first, order.cpu(), tiles), (first, order, tiles.cpu())]
            for other in others:
                with pytest.raises(AssertionError):
                    call(table, **{**arrays, name: other})
        with pytest.raises(AssertionError):                  # every other byte of an array
            call(table, **{**arrays, "workspace": workspace.repeat(2)[::2]})
    for other in (dict(starts=starts.cpu()), dict(which=which.cpu()), dict(first=first.cpu()), dict(order=order.cpu()), dict(tiles=tiles.cpu())):
        with pytest.raises(AssertionError):
            qb.qblora_adapter_groups(**{**dict(starts=starts, which=which, count=table.count, T=b.T), **other})

    w = [torch.zeros(5, device=au.DEV)]
    lst = qb.qblora_adamw_list([None], w, w, w, master=w)
    for at in range(4):
        lists = [[t.cpu()] if i == at else w for i, t in enumerate(w * 4)]
        with pytest.raises(AssertionError):
            qb.qblora_adamw_list([None], *lists[:3], master=lists[3])
    room = torch.empty(lst.norm_bytes, dtype=torch.uint8)
    for call in (lambda: qb.qblora_grad_norm(lst, 1.0, workspace=room), lambda: qb.qblora_grad_norm(lst, 1.0, out=torch.empty(2)),
                 lambda: qb.qblora_adamw_step(lst, torch.ones(1, dtype=torch.int64), 1e-3),
                 lambda: qb.qblora_adamw_step(lst, 1, torch.ones(1)), lambda: qb.qblora_adamw_step(lst, 1, 1e-3, clip=torch.ones(2))):
        with pytest.raises(AssertionError):
            call()


# ---- streams and graphs --------------------------------------------------------------------------------------

def test_captured_steps(qb):
    """Groups, forward and backward in one graph, replayed on other batches of the same size with eager work between."""
    b = au.Batch(50, 512, 256, 2, 2, [32, 64], [30, 1, 20, 4], [0, 1, 1, -1])
    grads = b.grads()
    table = b.table(qb, grads=grads)
    starts, which = au.dev(b.starts), au.dev(b.which)
    X, Y0, dY, dX0 = (au.dev_bf16(t) for t in (b.X, b.Y, b.dY, b.dX))
    Y, dX = Y0.clone(), dX0.clone()

    def step():
        Y.copy_(Y0)
        dX.copy_(dX0)
        groups = qb.qblora_adapter_groups(starts, which, 2, b.T)
        saved = torch.empty(qb.qblora_adapters_saved_bytes(table, b.T), dtype=torch.uint8, device=au.DEV)
        qb.qblora_adapters_fwd(table, groups, X, Y, saved=saved)
        qb.qblora_adapters_bwd(table, groups, X, dY, dX=dX, saved=saved)

    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for which_now in ([0, 1, 1, -1], [1, 1, 0, 0], [-1, -1, -1, 1], [0, 0, 0, 0]):
        which.copy_(au.dev(which_now))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (Y, dX, *(t for g in grads for t in g))]
        for t in (Y, dX, *(t for g in grads for t in g)):
            t.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip((Y, dX, *(t for g in grads for t in g)), want)), which_now


def test_two_streams(qb):
    """Two calls at once with workspaces of their own, on one table."""
    b = au.Batch(*LAYERS[5])
    table, groups = b.table(qb), b.groups(qb)
    X, Y = au.dev_bf16(b.X), au.dev_bf16(b.Y)
    want = qb.qblora_adapters_fwd(table, groups, X, Y.clone())
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [Y.clone() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for st, out in zip(streams, outs):
            with torch.cuda.stream(st):
                out.copy_(Y)
                qb.qblora_adapters_fwd(table, groups, X, out)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
