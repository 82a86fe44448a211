"""A workspace made for a number of tokens takes every smaller call: the block
over both kinds of cache, decoder layers and the MoE layer."""
import numpy as np
import pytest
import torch

from paper_2506_23635_gb300 import inputs as gen
from tests import paged_ref as ref
from tests.gpu_util import dev, need_gpu

pytestmark = pytest.mark.gpu


def moe():
    need_gpu()
    from paper_2506_23635_gb300 import moe as m
    return m


def _up(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


class Call:
    def __init__(self, m, D, hq, hkv, T):
        self.m, self.T = m, T
        self.c = ref.call(hq, hkv, 64, [(0, 0, T - 3), (1, 5, 1), (2, 100, 2)], seed=T)
        self.a = m.sa_dims(D, hq, hkv, 128, self.c["base"])
        shape = gen.AttnShape(D, hq, hkv, 128, self.c["base"], "bf16")
        self.w = [dev(t, "bf16") for t in gen.host_attn_weights(shape, 3)]
        self.x = _up((self.c["rng"].normal(size=(T, D))).astype(np.float32))
        self.seq, self.pos = _up(self.c["seq"]), _up(self.c["pos"])

    def paged_cache(self):
        c = self.c
        return self.m.PagedCache(_up(c["k"]).view(torch.float8_e4m3fn), _up(c["v"]).view(torch.float8_e4m3fn),
                                 _up(c["ks"]), _up(c["vs"]), _up(c["table"]))

    def slab(self):
        shape = (3, self.c["hkv"], max(int(self.c["pos"].max()) + 1, 8), 128)
        return [torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]


# (heads, a number of tokens, a smaller one): the smaller call splits its
# sequences into more parts a token than the larger
SIZES = [(48, 8, 257, 256), (8, 1, 70, 68), (8, 1, 2049, 2048)]


@pytest.mark.parametrize("hq,hkv,most,T", SIZES, ids=str)
@pytest.mark.parametrize("kind", ["paged", "slab"])
def test_attention_block_in_a_larger_calls_workspace(kind, hq, hkv, most, T):
    m = moe()
    call = Call(m, 512, hq, hkv, T)
    size = m.paged_sa_workspace_size if kind == "paged" else m.sa_workspace_size
    got = []
    for n in (T, most):
        ws = torch.empty(size(call.a, n), dtype=torch.uint8, device="cuda")
        x = call.x.clone()
        if kind == "paged":
            m.paged_sa_forward(call.a, call.paged_cache(), x, *call.w, call.seq, call.pos, ws=ws)
        else:
            m.sa_forward(call.a, x, *call.w, call.seq, call.pos, *call.slab(), ws=ws)
        got.append(x)
    assert m.get_last_error() == 0
    assert torch.equal(*got)


@pytest.mark.parametrize("T,most", [(64, 65), (64, 100), (24, 70)])
def test_layer_in_a_larger_calls_workspace(T, most):
    m = moe()
    L = gen.host_layer(gen.LayerShape(512, 1024, 8, 2, "bf16"), T, 7)
    t = [dev(a, "bf16") for a in (L.x, L.w_r, L.w1, L.v1, L.w2)]
    d = m.dims(512, 1024, 8, 2)
    got = [m.layer_forward(d, *t, ws=torch.empty(m.workspace_size(d, n), dtype=torch.uint8, device="cuda"))
           for n in (T, most)]
    assert m.get_last_error() == 0
    assert torch.equal(*got)
