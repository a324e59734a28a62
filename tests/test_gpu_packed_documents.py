"""Many rows of several packed documents, which are unpacked one after another."""
import numpy as np
import pytest
import torch

from tests.test_gpu_packed import SHAPES, bound, document, models, queries  # noqa: F401
from tests.test_gpu_packed_long import reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,docs", [
    ("dh128", [(1500, 600), (70, 3), (900, 700)]),
    ("dh64", [(3000, 1500), (4000, 1200), (1, 1)]),
])
def test_many_rows_of_several_documents(models, shape, docs):  # noqa: F811
    dh, H, G = SHAPES[shape]
    m = models(shape, "bf16")
    made = [document(m, 3 * i + n, n, shape, "bf16") for i, (n, _) in enumerate(docs)]
    pos = [np.arange(n - R, n) for n, R in docs]
    pos[0][:2] = -1
    r = m.rows([(d[0], p) for d, p in zip(made, pos)])
    q = queries(1, r.n, H, dh, "bf16")
    out = torch.full_like(q, float("nan"))
    before = m.launches()
    r.attention(1, q, out)
    assert m.launches() - before >= 5  # the few rows', two unpackings, two attentions
    i = 0
    for (doc, k, v), p in zip(made, pos):
        x = slice(i, i + len(p))
        ref, vmax, smax = reference(q[x], p, torch.from_numpy(k[:, 1]).cuda(),
                                    torch.from_numpy(v[:, 1]).cuda())
        err = np.abs((out[x].double() - ref).cpu().numpy()) - bound(
            "bf16", ref.cpu().numpy(), vmax.cpu().numpy()[..., 0], smax.cpu().numpy()[..., 0])
        assert not (err > 0).any(), float(err.max())
        i += len(p)
    assert torch.isfinite(out).all() and (out[:2] == 0).all()
    r.close()
    for d, _, _ in made:
        d.close()
