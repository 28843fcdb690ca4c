"""A drafter context for the cache operators' tests, and a cache beside its oracle (test helpers)."""
import numpy as np
import torch

from oracle import kv8 as o8
from paper_2609_09338_gb300 import binding as ob
from paper_2609_09338_gb300.workloads import DrafterShape

THETA = 1e6


def make_ctx(Hq, Hkv, hd, L=1):
    sh = DrafterShape(d_model=256, n_layers=L, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=hd, ffn_dim=256, vocab=256,
                      feat_dim=256, rope_theta=THETA)
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    d, a = sh.d_model, Hq * hd
    w = {"W_c": z(d, 256), "embed": z(256, d), "final_norm": z(d), "lm_head": z(256, d)}
    for k, s in {"attn_norm": (d,), "W_qkv": (sh.qkv_rows, 2 * d), "W_o": (d, a), "ffn_norm": (d,),
                 "W_gate": (256, d), "W_up": (256, d), "W_down": (d, 256)}.items():
        w[k] = [z(*s) for _ in range(L)]
    return ob.osprey_create(sh, w)


def table(B, max_pages, seed, spare=3):
    n = B * max_pages + spare
    return np.random.default_rng(seed).permutation(n)[:B * max_pages].reshape(B, max_pages).astype(np.int32), n


def rows(gen, shape, dtype, width=None):
    """Random rows [..., Hkv, hd], dense or as a view into rows of `width` elements."""
    *lead, H, hd = shape
    if width is None:
        return torch.randn(shape, generator=gen, device="cuda").to(dtype)
    wide = torch.randn((*lead, width), generator=gen, device="cuda").to(dtype)
    return wide[..., width - H * hd:].unflatten(-1, (H, hd))


class Model:
    """The rows of every sequence as bf16 values, and what the cache has to hold for them."""

    def __init__(self, L, B):
        self.k = [[[] for _ in range(B)] for _ in range(L)]
        self.v = [[[] for _ in range(B)] for _ in range(L)]

    def append(self, n, k, v):
        """k, v: float64 arrays [L, total, Hkv, hd] of the values cached."""
        r = 0
        for b, m in enumerate(n):
            for l in range(len(self.k)):
                self.k[l][b] += list(k[l, r:r + m])
                self.v[l][b] += list(v[l, r:r + m])
            r += m

    def check(self, kv, lens):
        """Codes and scales of finished pages and the tail's rows, bit for bit."""
        tab = kv.page_table.cpu().numpy()
        T = kv.tail_pages
        k8, v8 = kv.k8.cpu().numpy(), kv.v8.cpu().numpy()
        ks, vs = kv.k_scale.cpu().numpy(), kv.v_scale.cpu().numpy()
        kt, vt = kv.k_tail.double().cpu().numpy(), kv.v_tail.double().cpu().numpy()
        for l in range(len(self.k)):
            for b, n in enumerate(lens):
                for x, code, scale, tail, place in ((self.k, k8, ks, kt, o8.place_k), (self.v, v8, vs, vt, o8.place_v)):
                    x = np.array(x[l][b][:n])
                    for p in range(n // 16):
                        for h in range(x.shape[1]):
                            c, s = o8.encode_block(x[p * 16:p * 16 + 16, h])
                            np.testing.assert_array_equal(scale[l, tab[b, p], h], np.float32(s), err_msg=f"{l} {b} {p} {h}")
                            np.testing.assert_array_equal(code[l, tab[b, p], h], place(c), err_msg=f"{l} {b} {p} {h}")
                    last = (n - 1) // 16 if n else -1
                    for p in range(max(0, last - T + 1), last + 1):
                        m = min(16, n - p * 16)
                        got = tail[l, b * T + p % T, :, :m].transpose(1, 0, 2)
                        np.testing.assert_array_equal(got, x[p * 16:p * 16 + m], err_msg=f"{l} {b} {p}")
