"""What the forward point's calls refuse on CUDA tensors, before anything is enqueued."""
import pytest
import torch

from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward as F
from paper_2609_38095_gb300 import zo

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


def heads(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def ints(*v, dtype=torch.int64):
    return torch.tensor(v, dtype=dtype, device="cuda")


def rotate(**kw):
    args = dict(q=heads(4, 2, 64), k=heads(4, 1, 64), table=F.rotary_table(8, 64), positions=ints(0, 1, 2, 3)) | kw
    q, k = args.pop("q"), args.pop("k")
    return F.rotate_heads(q, k, **args)


@pytest.mark.parametrize("error,make", [
    (TypeError, lambda: {"q": heads(4, 2, 64).cpu()}), (TypeError, lambda: {"q": None}), (TypeError, lambda: {"q": heads(4, 2, 64, dtype=torch.float64)}),
    (ValueError, lambda: {"q": heads(8, 64)}), (ValueError, lambda: {"q": heads(4, 64, 2).transpose(1, 2)}),
    (TypeError, lambda: {"k": heads(4, 1, 64, dtype=torch.float16)}), (ValueError, lambda: {"k": heads(3, 1, 64)}), (ValueError, lambda: {"k": heads(4, 1, 32)}),
    (TypeError, lambda: {"table": heads(8, 64)}), (ValueError, lambda: {"table": F.rotary_table(8, 64)[:, ::2]}),
    (ValueError, lambda: {"table": F.rotary_table(8, 64)[0]}), (zo.ZoError, lambda: {"table": F.rotary_table(8, 128)}),
    (TypeError, lambda: {"positions": ints(0, 1, 2, 3).float()}), (ValueError, lambda: {"positions": ints(0, 1)}),
    (ValueError, lambda: {"layout": "other"}), (ValueError, lambda: {"q_weight": heads(63)}), (TypeError, lambda: {"k_weight": ints(1)}),
    (ValueError, lambda: {"k": None, "k_weight": heads(64)}), (ValueError, lambda: {"slots": ints(0, 1, 2, 3)}),
    (ValueError, lambda: {"slots": ints(0, 1), "k_out": heads(9, 1, 64)}), (TypeError, lambda: {"slots": ints(0, 1, 2, 3, dtype=torch.int32),
                                                                                "k_out": heads(9, 1, 64)}),
    (ValueError, lambda: {"q_out": heads(4, 3, 64)}), (ValueError, lambda: {"q_out": heads(5, 2, 64)}), (zo.ZoError, lambda: {"eps": -1.0}),
    (ValueError, lambda: {"v_out": heads(4, 1, 64)}),
])
def test_rotate_heads(error, make):
    kw = make()
    with pytest.raises(error):
        rotate(**kw)


def test_caches_of_unlike_rows():
    k = heads(4, 1, 64)
    with pytest.raises(ValueError):
        F.rotate_heads(heads(4, 2, 64), k, k, table=F.rotary_table(8, 64), positions=ints(0, 1, 2, 3), slots=ints(0, 1, 2, 3),
                       k_out=heads(2, 8, 1, 64), v_out=heads(4, 4, 1, 64))


def attend(**kw):
    args = dict(q=heads(4, 2, 64), k=heads(5, 1, 64), v=heads(5, 1, 64), spans=torch.zeros(3, 4, dtype=torch.int32, device="cuda")) | kw
    return F.attention(args.pop("q"), args.pop("k"), args.pop("v"), args.pop("spans"), **args)


@pytest.mark.parametrize("error,make", [
    (TypeError, lambda: {"k": heads(5, 1, 64).cpu()}), (TypeError, lambda: {"v": heads(5, 1, 64, dtype=torch.float16)}), (ValueError, lambda: {"v": heads(6, 1, 64)}),
    (ValueError, lambda: {"k": heads(5, 3, 64), "v": heads(5, 3, 64)}), (ValueError, lambda: {"k": heads(5, 0, 64), "v": heads(5, 0, 64)}),
    (ValueError, lambda: {"k": heads(5, 1, 32), "v": heads(5, 1, 32)}), (TypeError, lambda: {"spans": ints(0)}),
    (ValueError, lambda: {"spans": torch.zeros(2, 4, dtype=torch.int32, device="cuda")}), (ValueError, lambda: {"out": heads(4, 2, 32)}),
    (ValueError, lambda: {"slopes": torch.zeros(3, device="cuda")}), (TypeError, lambda: {"slopes": heads(2)}), (zo.ZoError, lambda: {"softcap": -1.0}),
    (zo.ZoError, lambda: {"scale": float("nan")}), (TypeError, lambda: {"scale": "large"}),
    (zo.ZoError, lambda: {"q": heads(4, 2, 264), "k": heads(5, 1, 264), "v": heads(5, 1, 264)}),
])
def test_attention(error, make):
    kw = make()
    with pytest.raises(error):
        attend(**kw)


def decode(**kw):
    args = dict(q=heads(2, 2, 64), k=heads(9, 8, 1, 64), v=heads(9, 8, 1, 64),
                pages=torch.zeros(2, 3, dtype=torch.int32, device="cuda"), lengths=ints(3, 4, dtype=torch.int32)) | kw
    return F.decode_attention(args.pop("q"), args.pop("k"), args.pop("v"), args.pop("pages"), args.pop("lengths"), **args)


@pytest.mark.parametrize("error,make", [
    (ValueError, lambda: {"k": heads(9, 8, 64), "v": heads(9, 8, 64)}), (ValueError, lambda: {"v": heads(9, 7, 1, 64)}),
    (TypeError, lambda: {"pages": ints(0, 0)}), (ValueError, lambda: {"pages": torch.zeros(3, 3, dtype=torch.int32, device="cuda")}),
    (ValueError, lambda: {"pages": torch.zeros(3, 2, dtype=torch.int32, device="cuda").T}), (TypeError, lambda: {"lengths": ints(3, 4)}),
    (ValueError, lambda: {"lengths": ints(3, dtype=torch.int32)}), (ValueError, lambda: {"k": heads(9, 0, 1, 64), "v": heads(9, 0, 1, 64)}),
])
def test_decode_attention(error, make):
    kw = make()
    with pytest.raises(error):
        decode(**kw)


@pytest.mark.parametrize("error,make", [
    (ValueError, lambda: ((heads(4, 2, 64), ints(0, 1, 2, 3)), {})), (TypeError, lambda: ((heads(4, 64), ints(0, 1, 2, 3).half()), {})),
    (ValueError, lambda: ((heads(4, 64), ints(0, 1, 2)), {})), (ValueError, lambda: ((heads(64, 4).T, ints(0, 1, 2, 3)), {})),
    (ValueError, lambda: ((heads(4, 64), ints(0, 1, 2, 3)), {"add": True})), (TypeError, lambda: ((heads(4, 64), ints(0, 1, 2, 3)), {"out": heads(1)})),
    (ValueError, lambda: ((heads(4, 64), ints(0, 1, 2, 3)), {"out": torch.zeros(2, device="cuda")})),
    (ValueError, lambda: ((heads(4, 64), ints(0, 1, 2, 3)), {"dtype": torch.float16})), (zo.ZoError, lambda: ((heads(4, 0), ints(0, 1, 2, 3)), {})),
])
def test_token_loss(error, make):
    args, kw = make()
    with pytest.raises(error):
        F.token_loss(*args, **kw)


def test_gradients_are_refused_where_torch_would_record_one():
    q = heads(4, 2, 64).requires_grad_(True)
    for call in (lambda: rotate(q=q), lambda: attend(q=q), lambda: decode(q=heads(2, 2, 64).requires_grad_(True)),
                 lambda: F.token_loss(heads(4, 64).requires_grad_(True), ints(0, 1, 2, 3)),
                 lambda: rotate(q_weight=heads(64).requires_grad_(True))):
        with pytest.raises(RuntimeError, match="gradient"):
            call()
        with torch.no_grad():
            call()


def test_spans_and_table():
    starts = ints(0, 3, dtype=torch.int32)
    for error, args, kw in ((TypeError, (ints(0, 3),), {"tokens": 3}), (ValueError, (starts, ints(0, 1, 2, dtype=torch.int32)), {"tokens": 3}),
                            (ValueError, (starts, None, ints(1, 2, dtype=torch.int32)), {"tokens": 3})):
        with pytest.raises(error):
            F.document_spans(*args, **kw)
    with pytest.raises(zo.ZoError):
        F.rotary_table(4, 7)
    with pytest.raises(zo.ZoError):
        F.rotary_table(4, 8, scale=0.0)
