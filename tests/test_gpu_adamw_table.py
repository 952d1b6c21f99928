"""The table of an AdamW step's tensors: what the step writes is listed once."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2010_16165_b200 import binding
    return binding


def tensor(bits, n=300):
    new = lambda k, dt=torch.float32: torch.zeros(k, device="cuda", dtype=dt)   # noqa: E731
    if bits == 32:
        return dict(p=new(n), g=new(n), m=new(n), v=new(n))
    return dict(p=new(n), g=new(n), m=new(n, torch.uint8), v=new(n, torch.uint8), m_scale=new(2), v_scale=new(2))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_tensor_that_is_listed_twice(B, bits):
    a, b = tensor(bits), tensor(bits)
    for key in a:
        with_shared = dict(b, **{key: a[key]})
        if key == "g":                                   # a gradient may be shared
            B.fp_adamw_step(B.fp_adamw_tensors([a, with_shared]), lr=1e-3)
        else:
            with pytest.raises(ValueError):
                B.fp_adamw_tensors([a, with_shared])
    with pytest.raises(ValueError):
        B.fp_adamw_tensors([a, a])
    with pytest.raises(ValueError):
        B.fp_adamw_tensors([a, dict(b, g=a["p"])])
    torch.cuda.synchronize()


def test_masks_may_be_shared_and_are_not_written(B):
    a, b = tensor(32), tensor(8)
    mask = torch.ones(3, device="cuda", dtype=torch.uint8)
    B.fp_adamw_step(B.fp_adamw_tensors([dict(a, mask=mask), dict(b, mask=mask)]), lr=1e-3)
    with pytest.raises(ValueError):
        B.fp_adamw_tensors([a, dict(b, mask=b["m"])])
    e = torch.empty(0, device="cuda")                    # tensors without elements share what they like
    B.fp_adamw_step(B.fp_adamw_tensors([a, dict(p=e, g=e, m=e, v=e), dict(p=e, g=e, m=e, v=e)]), lr=1e-3)
    torch.cuda.synchronize()
