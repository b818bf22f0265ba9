"""What the embedding, verification and distillation entry points refuse on the host, before
anything is launched (CPU: the C ABI with made-up addresses, the binding with host tensors)."""

import ctypes
import math

import pytest
import torch

import paper_2604_08706_amd as rbp
from paper_2604_08706_amd import _binding as b

NULL, P, ODD = ctypes.c_void_p(0), ctypes.c_void_p(4096), ctypes.c_void_p(4097)
BIG = 1 << 40


def _embed_fwd(table=P, tokens=P, seq=NULL, T=4, d=16, V=10, scale=1.0, out=P):
    return b.lib().policy_embed_fwd(table, tokens, seq, T, d, V, scale, out, NULL)


def _embed_bwd(dx=P, typ=rbp.RBP_F32, tokens=P, seq=NULL, T=4, d=16, V=10, scale=1.0, dW=P, acc=1,
               ws=P, ws_bytes=BIG):
    return b.lib().policy_embed_bwd(dx, typ, tokens, seq, T, d, V, scale, dW, acc, ws, ws_bytes,
                                    NULL)


def _verify(z=P, zd=P, typ=rbp.RBP_BF16, ld=10, ldd=10, x=P, n=NULL, u=P, B=2, K=3, V=10, tau=1.0,
            tok=P, lp=P, n_out=P, ws=P, ws_bytes=BIG):
    return b.lib().policy_verify_drafts(z, zd, typ, ld, ldd, x, n, u, B, K, V, tau, tok, lp, n_out,
                                        ws, ws_bytes, NULL)


def _distill(z=P, typ=rbp.RBP_F32, ld=10, ids=P, lt=P, mass=NULL, seq=P, length=P, T=4, V=10, K=3,
             B=2, n_seq=2, tau=1.0, scale=1.0, kl=P, loss=P, stats=P, dz=P, ws=P, ws_bytes=BIG):
    return b.lib().policy_distill_fwd_bwd(z, typ, ld, ids, lt, mass, seq, length, T, V, K, B, n_seq,
                                          tau, scale, kl, loss, stats, dz, ws, ws_bytes, NULL)


REFUSED = [
    (_embed_fwd, rbp.RBP_EINVAL, [dict(table=NULL), dict(tokens=NULL), dict(out=NULL), dict(T=-1),
                                  dict(d=0), dict(V=0), dict(scale=math.inf),
                                  dict(scale=math.nan)]),
    (_embed_fwd, rbp.RBP_EUNSUPPORTED, [dict(d=12), dict(table=ctypes.c_void_p(4104)),
                                        dict(out=ctypes.c_void_p(4098)), dict(T=1 << 31),
                                        dict(T=(1 << 30) + 1, d=128)]),
    (_embed_bwd, rbp.RBP_EINVAL, [dict(dx=NULL), dict(tokens=NULL), dict(dW=NULL), dict(T=-1),
                                  dict(d=0), dict(V=0), dict(typ=2), dict(typ=-1),
                                  dict(scale=math.nan), dict(dW=NULL, T=0), dict(ws=ctypes.c_void_p(4104))]),
    (_embed_bwd, rbp.RBP_EUNSUPPORTED, [dict(d=20), dict(dx=ctypes.c_void_p(4100)),
                                        dict(dW=ctypes.c_void_p(4104)), dict(T=(1 << 30) + 1)]),
    (_embed_bwd, rbp.RBP_EWORKSPACE, [dict(ws=NULL), dict(ws_bytes=0), dict(ws_bytes=64)]),
    (_verify, rbp.RBP_EINVAL, [dict(z=NULL), dict(x=NULL), dict(u=NULL), dict(tok=NULL),
                               dict(lp=NULL), dict(n_out=NULL), dict(B=-1), dict(K=-1), dict(V=0),
                               dict(ld=9), dict(ldd=9), dict(typ=7), dict(tau=0.0), dict(tau=-1.0),
                               dict(tau=math.inf), dict(tau=math.nan), dict(tau=1e-38), dict(tau=1e38),
                               dict(z=ODD), dict(zd=ODD), dict(ws=ODD),
                               dict(typ=rbp.RBP_F32, z=ctypes.c_void_p(4098))]),
    (_verify, rbp.RBP_EUNSUPPORTED, [dict(K=256), dict(B=1 << 23), dict(K=0, B=(1 << 21) + 1)]),
    (_verify, rbp.RBP_EWORKSPACE, [dict(ws=NULL), dict(ws_bytes=0)]),
    (_distill, rbp.RBP_EINVAL, [dict(z=NULL), dict(ids=NULL), dict(lt=NULL), dict(seq=NULL),
                                dict(length=NULL), dict(kl=NULL), dict(loss=NULL),
                                dict(stats=NULL), dict(T=-1), dict(V=0), dict(K=0), dict(B=0),
                                dict(n_seq=0), dict(ld=9), dict(typ=2), dict(tau=0.0),
                                dict(tau=math.nan), dict(tau=1e-38), dict(tau=1e38), dict(scale=math.inf),
                                dict(z=ODD), dict(ws=ctypes.c_void_p(4100)),
                                dict(dz=ctypes.c_void_p(4098))]),
    (_distill, rbp.RBP_EUNSUPPORTED, [dict(K=257), dict(T=1 << 31), dict(T=1 << 22)]),
    (_distill, rbp.RBP_EWORKSPACE, [dict(ws=NULL), dict(ws_bytes=7)]),
]


@pytest.mark.parametrize("call,status,args",
                         [(c, s, a) for c, s, all_ in REFUSED for a in all_],
                         ids=lambda v: v.__name__ if callable(v) else str(v))
def test_refused_on_the_host(call, status, args):
    assert call(**args) == status
    assert b.lib().rbp_last_error() != b""


def test_nothing_to_do_is_no_error():
    """No launch: there is no GPU here."""
    assert _embed_fwd(T=0, table=NULL, tokens=NULL, out=NULL) == rbp.RBP_OK
    assert _embed_bwd(T=0, dx=NULL, tokens=NULL, ws=NULL, ws_bytes=0) == rbp.RBP_OK
    assert _verify(B=0, z=NULL, zd=NULL, x=NULL, u=NULL) == rbp.RBP_OK
    assert _distill(T=0, z=NULL, ids=NULL, kl=NULL, ws=NULL, ws_bytes=0) == rbp.RBP_OK
    assert b.lib().rbp_last_error() == b""


def _t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


def _calls(device="cpu"):
    def f(*shape, dtype=torch.float32):
        return torch.zeros(shape, dtype=dtype, device=device)

    i = torch.int32
    return {
        "embed_fwd": (rbp.policy_embed_fwd, dict(
            table=f(10, 8, dtype=torch.bfloat16), tokens=f(4, dtype=i), seq_of_token=f(4, dtype=i),
            out=f(4, 8, dtype=torch.bfloat16))),
        "embed_bwd": (rbp.policy_embed_bwd, dict(
            dx=f(4, 8), tokens=f(4, dtype=i), seq_of_token=f(4, dtype=i), dW=f(10, 8),
            ws=f(1 << 16, dtype=torch.uint8))),
        "verify": (rbp.policy_verify_drafts, dict(
            logits=f(2, 3, 10), draft_logits=f(2, 2, 10), draft_tokens=f(2, 2, dtype=i),
            n_draft=f(2, dtype=i), u=f(2, 3), out_tokens=f(2, 3, dtype=i), out_logp=f(2, 3),
            n_out=f(2, dtype=i), ws=f(1 << 16, dtype=torch.uint8))),
        "distill": (rbp.policy_distill_fwd_bwd, dict(
            logits=f(4, 10), teacher_ids=f(4, 2, dtype=i), teacher_logits=f(4, 2),
            teacher_lse=f(4), seq_of_token=f(4, dtype=i), seq_len=f(2, dtype=i) + 1, n_seq_total=2,
            kl=f(4), loss_accum=f(1), stats=f(2), dlogits=f(4, 10),
            ws=f(1 << 16, dtype=torch.uint8))),
    }


NAMES = sorted(_calls())


@pytest.mark.parametrize("name", NAMES)
def test_host_tensors_are_refused(name):
    call, args = _calls()[name]
    with pytest.raises(ValueError, match="device tensor"):
        call(**args)
    for key in args:
        if key in ("n_seq_total", "ws", "seq_of_token", "draft_logits", "n_draft", "teacher_lse",
                   "dlogits", "draft_tokens"):
            continue
        with pytest.raises((TypeError, ValueError, AttributeError)):
            call(**dict(args, **{key: [0] * 8}))


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_wrong_types_shapes_and_strides_are_refused(name):
    call, args = _calls("cuda")[name]
    call(**args)  # as it stands it is accepted
    torch.cuda.synchronize()
    for key, t in args.items():
        if key in ("n_seq_total", "ws"):
            continue
        wrong = t.to(torch.float64 if t.is_floating_point() else torch.int64)
        with pytest.raises(TypeError):
            call(**dict(args, **{key: wrong}))
        if t.numel() > 1 and key not in ("tokens", "seq_len"):  # (these give a size)
            with pytest.raises(ValueError):
                call(**dict(args, **{key: t.reshape(-1)[:-1]}))
        spread = torch.zeros(tuple(t.shape) + (2,), dtype=t.dtype, device="cuda")[..., 0]
        if t.dim() > 1 or t.numel() > 1:
            with pytest.raises(ValueError):
                call(**dict(args, **{key: spread}))
    with pytest.raises(rbp.RbpError) as e:
        if name == "embed_fwd":
            call(**dict(args, scale=math.inf))
        else:
            call(**dict(args, ws=args["ws"][:0]))
    assert e.value.status == (rbp.RBP_EINVAL if name == "embed_fwd" else rbp.RBP_EWORKSPACE)


@pytest.mark.gpu
def test_uneven_rows_and_mixed_types_are_refused():
    call, args = _calls("cuda")["verify"]
    wide = torch.zeros((2, 4, 12), device="cuda")
    with pytest.raises(ValueError, match="evenly"):  # sequences 48 apart, rows 12
        call(**dict(args, logits=wide[:, :3, :10]))
    with pytest.raises(TypeError, match="type of logits"):
        call(**dict(args, draft_logits=args["draft_logits"].bfloat16()))
    with pytest.raises(ValueError):
        call(**dict(args, logits=torch.zeros((1, 1, 10), device="cuda").expand(2, 3, 10)))
    call, args = _calls("cuda")["distill"]
    with pytest.raises(TypeError, match="type of logits"):
        call(**dict(args, dlogits=args["dlogits"].bfloat16()))
    with pytest.raises(ValueError, match="strides"):
        call(**dict(args, dlogits=torch.zeros((4, 12), device="cuda")[:, :10]))
    with pytest.raises(ValueError, match="evenly"):
        call(**dict(args, logits=torch.zeros((10, 4), device="cuda").t()))
