"""Causal attention at the edges of what its entry points take: offsets that are no list, sizes next to the limits, infinite keys, rows of many small weights, fp16
signals of very different sizes."""
import ctypes as C
import math
import struct

import pytest

from test_causal_attention import EUNSUPPORTED, U, U32, _A, _check, _dt, _ends, _lib, _reference, _shape, _tensors

gpu = pytest.mark.gpu


# ---- sizes (no GPU call is made) ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("seqs,T,Hq,status", [
    (1, (1 << 31) - 1, 1, EUNSUPPORTED), (1, (1 << 31) - 127, 1, EUNSUPPORTED), (1, (1 << 31) - 128, 1, EUNSUPPORTED), (1, 1 << 30, 2, EUNSUPPORTED),
    (1, 8323072 * 128 + 1, 1, EUNSUPPORTED), (1, 8323072 * 128, 1, 0), (8323072, 1, 1, 0), (8323073, 1, 1, EUNSUPPORTED), (8323072 // 4, 1, 4, 0)])
def test_sequences_of_one_length_at_the_limit(seqs, T, Hq, status):
    """8323072 tiles of 128 rows are what a launch takes; T + 127 may pass 31 bits."""
    lib, n = _lib(), C.c_size_t(0)
    D = 1
    s = _shape(seqs=seqs, T=T, rows=seqs * T, Hq=Hq, Hkv=1, D=D, offsets_type=0, ldq=Hq, ldk=1, ldv=1, ldo=Hq, head_q=1, head_k=1, head_v=1, head_o=1,
               lddo=Hq, lddq=Hq, lddk=1, lddv=1, head_do=1, head_dq=1, head_dk=1, head_dv=1)
    for backward in (0, 1):
        assert lib.abs_causal_attention_workspace_bytes(C.byref(s), backward, C.byref(n)) == status


@pytest.mark.parametrize("rows,seqs,Hq,status", [
    (8323071 * 128, 1, 1, 0), (8323072 * 128, 1, 1, EUNSUPPORTED), ((1 << 31) - 1, 1, 1, EUNSUPPORTED), (100, 8323072, 1, 0), (128, 8323072, 1, EUNSUPPORTED)])
def test_packed_sequences_at_the_limit(rows, seqs, Hq, status):
    lib, n = _lib(), C.c_size_t(0)
    s = _shape(seqs=seqs, rows=rows, Hq=Hq, Hkv=1, D=1, **{k + n: 1 for k in ("ld", "head_") for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")})
    for backward in (0, 1):
        assert lib.abs_causal_attention_workspace_bytes(C.byref(s), backward, C.byref(n)) == status


# ---- offsets that are no list -------------------------------------------------------------------------------------------

def _list_kernel_arguments(seqs, rows, offsets, out):
    """The kernels' parameters with what the list of tiles is made from: offsets of 32 bits, no sums of more than the list."""
    p = bytearray(512)
    struct.pack_into("<8i", p, 0, 0, 1, 1, 8, seqs, 0, 0, 0)           # type, Hq, Hkv, D, seqs, T, wide, zero_rest
    struct.pack_into("<qQQ", p, 32, rows, offsets, out)
    return (C.c_char * len(p)).from_buffer(p)


@gpu
@pytest.mark.parametrize("rows,full", [(1 << 20, (1 << 18) + 2), (1 << 22, 1 << 17), (1000, 300), (128, 40)])
def test_the_list_of_tiles_ends_where_its_room_does(rows, full):
    """Sequences that all have all rows, an empty one behind each: up to 2^32 tiles of which the list holds rows / 128 + sequences."""
    import torch
    lib, seqs = _lib(), 2 * full
    off = torch.tensor([0, rows] * full + [0], dtype=torch.int32, device="cuda")
    room, guard = rows // 128 + seqs, 4096
    buf = torch.full((room + 1 + 2 * guard, 2), -7, dtype=torch.int32, device="cuda")
    call = lib["_ZN4absk22launch_attention_tilesERKNS_10AttentionPEP12ihipStream_t"]
    p = _list_kernel_arguments(seqs, rows, off.data_ptr(), buf[guard].data_ptr())
    assert call(C.byref(p), C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    torch.cuda.synchronize()
    assert (buf[:guard] == -7).all() and (buf[-guard:] == -7).all()
    used, each = min(room, full * (-(-rows // 128))), -(-rows // 128)
    entries = buf[guard + 1:-guard].long()
    assert buf[guard].tolist() == [used, 0] and (entries[used:] == -7).all()
    entries = entries[:used]
    assert (entries[:, 0] % 2 == 0).all() and (entries[:, 0] >= 0).all() and (entries[:, 0] < seqs).all()
    # every sequence's tiles side by side, from its last to its first
    place = torch.arange(used, device="cuda")
    assert torch.equal(entries[:, 1], each - place % each)
    assert torch.equal(entries[:, 0], entries[place - place % each, 0])


@gpu
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f16", 24), ("f32", 40)])
def test_many_offsets_that_are_no_list_stay_inside(dtype, D):
    """More than 64 sequences, through the C entry points, with all that is written between guards."""
    import torch
    from paper_2406_13936_amd import binding as B
    lib, R, H = _lib(), 300, 2
    q, k, v, do = _tensors(R, H, H, D, dtype)
    e, ld = q.element_size(), H * D
    for bad in ([0, R] * 60, [-9, 5000] * 40, [R, 0] * 50, list(range(R, R - 100, -1)), [0] * 70 + [R], [(i * 7919) % 400 - 50 for i in range(129)]):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        s = _shape(type={"f32": 0, "bf16": 1, "f16": 2}[dtype], seqs=len(bad) - 1, Hq=H, Hkv=H, D=D, rows=R,
                   **{n: ld if n[0] == "l" else D for n in [f for f, _ in B.AttentionShape._fields_ if f[:2] == "ld" or f[:5] == "head_"]})
        guarded = []

        def room(nbytes):
            nbytes = (nbytes + 255) // 256 * 256
            t = torch.full((nbytes + 2048,), 0x5a, dtype=torch.uint8, device="cuda")
            guarded.append(t)
            return t[1024:].data_ptr()
        n = C.c_size_t(0)
        stream = torch.cuda.current_stream().cuda_stream
        o, lse = room(R * ld * e), room(H * R * 4)
        for zero_rest in (0, 1):
            assert lib.abs_causal_attention_workspace_bytes(C.byref(s), 0, C.byref(n)) == 0
            assert lib.abs_causal_attention(C.byref(s), q.data_ptr(), k.data_ptr(), v.data_ptr(), off.data_ptr(), 0.2, o, lse, zero_rest,
                                            room(n.value), n.value, stream) == 0
            assert lib.abs_causal_attention_workspace_bytes(C.byref(s), 1, C.byref(n)) == 0
            grads = [room(R * ld * e) for _ in range(3)]
            assert lib.abs_causal_attention_backward(C.byref(s), do.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o, lse, off.data_ptr(), 0.2,
                                                     *grads, zero_rest, room(n.value), n.value, stream) == 0
        torch.cuda.synchronize()
        for t in guarded:
            assert (t[:1024] == 0x5a).all() and (t[-1024:] == 0x5a).all()


# ---- infinite keys ------------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 100), ("f16", 80), ("f32", 48)])
@pytest.mark.parametrize("T", [2, 31, 32, 33, 63, 64, 65, 97, 130])
def test_infinite_keys_whose_scores_are_minus_infinity(T, dtype, D):
    """A key that every query that sees it scores with minus infinity has no weight in any row: its gradients are zeros whether or not its block of
    queries ends behind the sequence's last, as are others' with their key in its place."""
    import torch
    A = _A()
    q, k, v, do = _tensors(T + 40, 2, 1, D, dtype, T)
    off = torch.tensor([0, T, T + 40], dtype=torch.int32, device="cuda")
    c = D // 3
    q[..., c] = -q[..., c].abs() - 0.25
    for at in {T - 1, T // 2, max(1, T - 33)}:
        k2 = k.clone()
        k2[at, 0, c] = float("inf")
        o, lse = A.causal_attention(q, k2, v, offsets=off)
        assert torch.isfinite(o).all() and torch.isfinite(lse).all()
        dq, dk, dv = A.causal_attention_backward(do, q, k2, v, o, lse, offsets=off)
        assert (dk[at] == 0).all() and (dv[at] == 0).all()
        assert torch.isfinite(dk).all() and torch.isfinite(dv).all()
        # a query that sees it has 0 times infinity in one place
        others = [i for i in range(D) if i != c]
        assert torch.isfinite(dq[:, :, others]).all() and torch.isfinite(dq[:at]).all() and torch.isfinite(dq[T:]).all()
        # the same with the key far away instead: a score that leaves it no weight either
        k2[at, 0, c] = 30000.0
        o1, lse1 = A.causal_attention(q, k2, v, offsets=off)
        _, dk1, dv1 = A.causal_attention_backward(do, q, k2, v, o1, lse1, offsets=off)
        assert torch.equal(o1, o) and torch.equal(lse1, lse) and torch.equal(dk1, dk) and torch.equal(dv1, dv)


# ---- weights in 16 bits -------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("score,place", [(18.0, 0), (18.0, 77), (11.0, 0), (5.5, 200), (5.5, 4000), (20.0, 9000)])
def test_long_rows_that_one_key_dominates(score, place, dtype):
    """Weights e^-18 = 2^-26 of the largest add up to 2^-11 of o over tens of thousands of keys.  In fp16 they are held times 2^7, so that one is off by half
    a step, 2^-25, of that: by 2^-32 of the largest weight, and a key that comes 2^7.9 above the reference is at most 2^15."""
    import torch
    A = _A()
    T, D, dt = 32768, 16, _dt(dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k = (torch.randn((T, h, D), device="cuda", generator=gen).to(dt) for h in (2, 1))
    v = (1 + 0.1 * torch.randn((T, 1, D), device="cuda", generator=gen)).to(dt)
    q[..., 0], q[..., 1:], k[..., 0] = 1, 0, 0       # scores are 0, exactly, but of one key
    k[place, 0, 0], v[place] = score, 0
    o, lse = A.causal_attention(q, k, v, scale=1.0)
    u = 0.0 if dtype == "f32" else U[dtype]
    for i in (0, 63, 64, 300, 4001, 9010, 20001, T - 1):
        s = torch.zeros(i + 1, dtype=torch.float64, device="cuda")
        if place <= i:
            s[place] = score
        p, top, vv = torch.softmax(s, 0), torch.logsumexp(s, 0), v[:i + 1, 0].double()
        rel = (D + 4) * U32 * score + 8 * U32 * (1 + score + float(top))
        err = (u + 4 * rel + (i + 9) * U32) * (p @ vv.abs()) + (2.0 ** -32 * vv.abs().sum(0) if dtype == "f16" else 0)
        want = p @ vv
        off = err + U[dtype] * (want.abs() + err) + (2.0 ** -25 if dtype == "f16" else 0)
        for h in range(2):
            _check(o[i, h], want.cpu(), off.cpu(), (i, h))
            assert abs(float(lse[h, i]) - float(top)) <= 2 * rel + (i + 9) * U32 + 4 * U32 * float(top)


@gpu
@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("D", [40, 64, 75, 128])
def test_fp16_gradients_of_a_sequence_and_head_do_not_depend_on_others(D, many):
    """Signals and values 2^25 apart: what one sequence, or one group of heads, has in a call is what it has alone, to the bit."""
    import torch
    A = _A()
    lens = [70, 1, 0, 200, 129, 64] + ([3, 0] * 40 if many else [])
    ends, Hq, Hkv = _ends(lens), 4, 2
    q, k, v, do = _tensors(ends[-1], Hq, Hkv, D, "f16", D)
    factor = [2.0 ** 9, 1.0, 1.0, 2.0 ** -12, 2.0 ** -3, 2.0 ** 3]
    for i, f in enumerate(factor):
        do[ends[i]:ends[i + 1]] *= f
        v[ends[i]:ends[i + 1]] *= f ** 0.25
    do[:, 2:] *= 2.0 ** 4
    v[:, 1] *= 2.0 ** 2
    off = torch.tensor(ends, device="cuda")
    o, lse = A.causal_attention(q, k, v, offsets=off)
    grads = A.causal_attention_backward(do, q, k, v, o, lse, offsets=off)
    for i in range(6):
        a, e = ends[i], ends[i + 1]
        if a == e:
            continue
        alone = A.causal_attention_backward(do[a:e], q[a:e], k[a:e], v[a:e], o[a:e], lse[:, a:e].contiguous())
        assert all(torch.equal(g[a:e], t) for g, t in zip(grads, alone)), i
        for g in range(Hkv):
            hq, hk = slice(2 * g, 2 * g + 2), slice(g, g + 1)
            alone = A.causal_attention_backward(do[a:e, hq], q[a:e, hq], k[a:e, hk], v[a:e, hk], o[a:e, hq], lse[hq, a:e].contiguous())
            assert all(torch.equal(t[a:e, h], x) for t, h, x in zip(grads, (hq, hk, hk), alone)), (i, g)
        assert all((g[a:e] != 0).any() for g in grads) or e - a == 1
    # and they are right: small signals keep their bits beside large ones
    a, e = ends[3], ends[4]
    want, err = _reference(q[a:e], k[a:e], v[a:e], [0, e - a], 1 / math.sqrt(D), "f16", do[a:e], o[a:e], lse[:, a:e])
    for g, n in zip(grads, ("dq", "dk", "dv")):
        _check(g[a:e], want[n], err[n], n)
