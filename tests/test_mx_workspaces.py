"""Workspaces of other types than bytes."""
import pytest

from paper_2602_17698_amd import binding as sb

torch = pytest.importorskip("torch")


@pytest.fixture()
def ctx():
    c = sb.Context(device=-1)               # no device: what passes all checks ends with ERR_HIP
    yield c
    c.close()


def no_device(call):
    with pytest.raises(sb.SbitsError) as e:
        call()
    assert e.value.status == sb.ERR_HIP


def test_workspaces_count_in_bytes(ctx):
    u8 = torch.uint8
    r, hidden, inner, tokens = sb.Router(experts=4, top_k=2), 64, 32, 3
    up = sb.mx(torch.zeros(4 * 2 * inner, hidden // 2, dtype=u8), torch.zeros(4 * 2 * inner, 4, dtype=u8), hidden)
    down = sb.mx(torch.zeros(4 * hidden, inner // 2, dtype=u8), torch.zeros(4 * hidden, 4, dtype=u8), inner)
    need = ctx.expert_layer_ws_bytes(r, tokens, up, down)
    space = torch.zeros(need + 256, dtype=u8)
    space = space[-space.data_ptr() % 256:][:need]
    x, out = torch.zeros(tokens, hidden, dtype=torch.bfloat16), torch.zeros(tokens, hidden, dtype=torch.bfloat16)
    args = (r, torch.zeros(tokens, 4), None, x, up, down, out, torch.zeros(tokens, 2, dtype=torch.int32), torch.zeros(tokens, 2))
    assert need % 4 == 0
    no_device(lambda: ctx.expert_layer(*args, space.view(torch.float32)))
    with pytest.raises(sb.SbitsError) as e:
        ctx.expert_layer(*args, space.view(torch.float32)[:-1])
    assert e.value.status == sb.ERR_WORKSPACE
