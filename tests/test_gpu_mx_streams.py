"""GPU: the streams a caller may name without having made one: the null stream, the legacy default stream and that of the calling thread."""
import threading

import numpy as np
import pytest

from oracle import mx as MX
from paper_2602_06079_amd import workloads as W
from tests.test_gpu_mx_product import device, operand, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stream", [0, 1, 2], ids=["null", "legacy", "per_thread"])
def test_default_streams(canz, stream):
    """Rounding, a product that rounds before, one that rounds on the way, the way back and the step with images; from the main thread and from another."""
    import torch
    m, n, k = 100, 300, 700
    rng = np.random.default_rng(stream)
    b = operand(rng, n, k, 2)
    db = device(b)
    vx = MX.values(*operand(rng, m, k, 2))
    x = torch.from_numpy(vx.astype(np.float32)).cuda()
    img = torch.empty(canz.canz_mx_image_bytes(m, k), dtype=torch.uint8, device="cuda")
    c, c1, back = torch.empty(m, n, device="cuda"), torch.empty(1, n, device="cuda"), torch.empty(m, k, device="cuda")
    products = [canz.MxProduct(m=m, n=n, k=k, a=[x], b=[db], c=[c], a_dtype=W.DT_F32, out_dtype=W.DT_F32),
                canz.MxProduct(m=1, n=n, k=k, a=[x], b=[db], c=[c1], a_dtype=W.DT_F32, out_dtype=W.DT_F32)]
    ws = workspace(canz, products)
    hp = canz.Hparams()
    w = torch.from_numpy(W.gen_param(1, 0, 64, 96)).cuda()
    step = canz.Group(rows=64, cols=96, grad=[torch.from_numpy(W.gen_grad(1, 0, 64, 96)[0]).cuda()], mom=[torch.zeros(64, 96, device="cuda")], out=[w],
                      grad_dtype=W.DT_F32, out_dtype=W.DT_F32)
    images = canz.MxImages(by_row=[torch.empty(canz.canz_mx_image_bytes(64, 96), dtype=torch.uint8, device="cuda")])
    step_ws = torch.empty(canz.canz_muon_workspace_bytes([step], hp), dtype=torch.uint8, device="cuda")
    want = MX.product(vx, MX.values(*b))
    failed = []

    def calls():
        try:
            canz.canz_mx_quantize([canz.MxGroup(rows=m, cols=k, mat=[x], by_row=[img])], MX.FLOOR, stream)
            canz.canz_mx_dequantize([canz.MxGroup(rows=m, cols=k, mat=[back], by_row=[img])], stream)
            canz.canz_mx_product(products, ws, ws.numel(), stream)
            canz.canz_muon_step_images([step], hp, [images], MX.FLOOR, step_ws, step_ws.numel(), stream)
        except Exception as e:
            failed.append(e)
    for other in (False, True):
        for t in (c, c1, back):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        if other:
            t = threading.Thread(target=calls)
            t.start()
            t.join()
        else:
            calls()
        torch.cuda.synchronize()
        assert not failed
        assert np.array_equal(c.double().cpu().numpy(), want) and np.array_equal(c1.double().cpu().numpy(), want[:1])
        assert np.array_equal(back.double().cpu().numpy(), vx)
        got = MX.unpack(images.by_row[0].cpu().numpy(), 64, 96)
        ref = MX.quantize(w.double().cpu().numpy(), MX.FLOOR)
        assert got[2] and np.array_equal(got[0], ref[0]) and np.array_equal(got[1], ref[1])
