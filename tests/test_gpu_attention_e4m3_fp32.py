"""An fp32 output of the attention over an e4m3 cache keeps the softmax numerators' 24 bits.

One token has weight exp(z) with -1 <= z < 0 and V = 1, one has z = 0 and V = 0, and all others are so
far below (exp2 of less than -300) that their weight is 0: the output is p / (1 + p), p = exp(z).
Every product q . k is a single exact term.  Relative error, in units of 2^-23:
  z      scale * log2(e) (its constant 1/4, its rounding 1/2) and z itself (1/2), times |z| <= 1    1.25
  exp2   one step                                                                                   1
  1 + p  (all other additions are of zeros)                                                         0.5
  p V    a numerator in parts adds up in at most three steps                                        3
  1 / (1 + p), and the product with it                                                              1.5
7.25 in all, below 2^-20.  (A numerator of 17 bits alone may be 2^-17 off.)"""
import numpy as np
import pytest
import torch

from paper_2606_08446_amd import sparrow as S

from parity import log

pytestmark = pytest.mark.gpu

DEV = "cuda"
D = 128


@pytest.fixture(autouse=True)
def _need_gpu(gpu_device):
    S.load()
    yield


# one workgroup per unit (few tokens, up to 8 query heads a KV head), streaming waves (16 query heads; a
# wide block table) and units that several waves share
@pytest.mark.parametrize("B,hq,hkv,ps,L,table", [(40, 8, 2, 16, 2, 1), (40, 16, 2, 32, 130, 5), (40, 16, 1, 16, 2, 1),
                                                 (24, 32, 2, 64, 200, 4), (24, 8, 2, 16, 90, 200), (3, 16, 1, 16, 5000, 313)])
def test_numerators_keep_24_bits(B, hq, hkv, ps, L, table):
    log(f"case e4m3 numerators B={B} heads={hq},{hkv} ps={ps} L={L}")
    g = np.random.default_rng(B + hq + ps + L)
    pages = -(-L // ps)
    P = B * pages
    bt = np.full((B, table), -1, np.int32)
    bt[:, :pages] = g.permutation(P).reshape(B, pages)
    k, v = np.zeros((P, hkv, ps, D), np.float32), np.zeros((P, hkv, ps, D), np.float32)
    k[..., 0] = 448.0
    kb = np.full((P, hkv, ps), 127 + 2)               # the far tokens' K is 1792
    for b in range(B):
        top, one = g.choice(L, 2, replace=False)
        at = bt[b, top // ps], slice(None), top % ps
        k[at], kb[at] = 0.0, 127
        at = bt[b, one // ps], slice(None), one % ps
        k[at], kb[at] = 0.0, 127
        k[at + (0,)] = 1.0
        v[at] = 1.0
    exps = np.full((P, hkv, ps // 4, 2, 4), 127, np.uint8)
    exps[:, :, :, 0] = kb.reshape(P, hkv, ps // 4, 4)
    k8, v8 = (torch.from_numpy(x).to(torch.float8_e4m3fn).to(DEV) for x in (k, v))
    q = torch.zeros((B, hq, D))
    q[..., 0] = -torch.from_numpy(g.uniform(1, 8, (B, hq))).to(torch.bfloat16).float()
    out = S.dense_decode_attn_e4m3(
        q.to(torch.bfloat16).to(DEV), k8, v8, torch.from_numpy(exps).to(DEV), torch.from_numpy(bt).to(DEV),
        torch.full((B,), L, dtype=torch.int32, device=DEV), scale=0.125)
    p = np.exp(0.125 * q[..., 0].double().numpy())[..., None]
    want = p / (1 + p)
    err = np.abs(out.cpu().double().numpy() - want) / want
    log(f"largest relative error {err.max():.3e}, 2^{np.log2(err.max()):.2f}")
    assert err.max() <= 2.0 ** -20
