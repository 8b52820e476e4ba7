"""The long sums of the relation head's backward: the bias gradient over key tiles that share a table,
and the norms' column gradients over many rows, each column against its own absolute sum."""
import numpy as np
import pytest

import paper_1906_07155_amd as rex
from gpu_helpers import log
from test_gpu_relation_attn import Case, f64
from test_gpu_relation_norm import Case as NormCase

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rex.lib()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,ragged", [((90, 3, 768, 1, 1, 8, 3), False), ((90, 3, 768, 4, 2, 16, 5), True),
                                          ((70, 33, 512, 6, 1, 72, 3), True)], ids=str)
def test_key_tiles_that_share_a_table(dtype, shape, ragged):
    """More key tiles than partial tables: a workgroup adds several of them up in one."""
    log("sums tables %s %s" % (dtype, shape))
    B, nq, nk, H, hkv, D, nb = shape
    rng = np.random.default_rng(7)
    lens = [int(n) for n in rng.integers(0, nk + 1, B)] if ragged else None
    c = Case(dtype, B, nq, nk, H, hkv, D, nb, k_len=lens, masked=0.1 if ragged else 0.0, seed=9)
    need = rex.box_attn_workspace_size(c.q, c.k, c.v, True, q_boxes=c.geo["q_boxes"], k_boxes=c.geo["k_boxes"], bias=c.geo["bias"])
    bare = rex.box_attn_workspace_size(c.q, c.k, c.v, True)
    one = B * H * nb * nb * 4                       # the images' tables of one run of key tiles
    tiles = nk // (32 if D <= 32 else 16)
    assert 0 < (need - bare) // one < tiles, "key tiles have a table each"   # (padding is less than one)
    c.check(c.both(), "shared tables")


def terms(c):
    """Every row's contribution to each column gradient, and what it is a sum of in absolute value."""
    a = {k: f64(v) if torch.is_tensor(v) else v for k, v in c.args.items()}
    x, b, gy, gu = f64(c.x), f64(c.branch), f64(c.gy), f64(c.gu)
    one, zero = np.ones(c.C), np.zeros(c.C)
    w1, w2 = (one if a[n] is None else a[n] for n in ("post_weight", "pre_weight"))
    c1 = zero if a["post_bias"] is None else a["post_bias"]
    gate = np.repeat(a["gate"], c.rows // c.gates, 0) * a["alpha"] if c.gates else a["alpha"]
    layer = a["norm"] == "layer"

    def hat(t, size):
        m = t.mean(1, keepdims=True) if layer else np.zeros((len(t), 1))
        rstd = 1 / np.sqrt(((t - m) ** 2).mean(1, keepdims=True) + a["eps"])
        return (t - m) * rstd, (size + np.abs(m)) * rstd, rstd

    h1, h1b, _ = hat(b, np.abs(b))
    z, zb = h1 * w1 + c1, h1b * np.abs(w1) + np.abs(c1)
    y, yb = x + gate * z, np.abs(x) + np.abs(gate) * zb
    h2, h2b, r2 = hat(y, yb)
    g, gb = gu * w2, np.abs(gu * w2)
    t = g - h2 * (g * h2).mean(1, keepdims=True) - (g.mean(1, keepdims=True) if layer else 0)
    d = gy + r2 * t
    db = np.abs(gy) + r2 * (gb + h2b * (gb * h2b).mean(1, keepdims=True) + gb.mean(1, keepdims=True))
    return {"gate": (d * z * a["alpha"], db * zb * abs(a["alpha"])), "post_weight": (d * gate * h1, db * np.abs(gate) * h1b),
            "post_bias": (d * gate, db * np.abs(gate)), "pre_weight": (gu * h2, np.abs(gu) * h2b), "pre_bias": (gu, np.abs(gu))}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C,gates,norm", [(513, 250, 1, "layer"), (2000, 128, 4, "rms"), (3000, 1024, 0, "layer"),
                                               (777, 77, 7, "layer"), (1500, 2056, 1, "rms")])
def test_column_gradients(dtype, rows, C, gates, norm):
    """A column is a binary32 sum: element by element its error is at most one rounding, 2^-24, of what
    is added up for each of its rows, and some 64 roundings of each term (two norms, their means of C
    terms in a tree, products); norm-wise these are independent, 2 sqrt(rows) + 64 of them with room.
    A reference without one of its rows, or with one twice, is told apart."""
    log("sums columns %s %d %d %d %s" % (dtype, rows, C, gates, norm))
    c = NormCase(dtype, rows, C, norm, gates, seed=5)
    got = c.both()
    for key, (each, size) in terms(c).items():
        if got[key] is None:
            continue
        parts = gates if key == "gate" else 1
        have = f64(got[key]).reshape(parts, C)
        want, big = (t.reshape(parts, -1, C).sum(1) for t in (each, size))
        err, n = np.abs(have - want), rows // parts
        assert np.all(err <= (n + 64) * 2.0 ** -24 * big), (key, (err / big).max() * 2 ** 24)
        near = (2 * np.sqrt(n) + 64) * 2.0 ** -24 * np.linalg.norm(big)
        assert np.linalg.norm(err) <= near, (key, np.linalg.norm(err) / near)
        for row in (0, n // 2, n - 1):              # each alone is more than the bound allows
            lost = want.copy()
            lost[0] -= each.reshape(parts, -1, C)[0, row]
            assert np.linalg.norm(have - lost) > near, (key, row)
