"""Making descriptors of the transformer-block calls: what does not fit its field or has no field is an error, not something else (CPU only)."""
import pytest

from paper_1902_04610_amd import salus
from paper_1902_04610_amd.salus import Pool

GATED = dict(job=0, M=4, K=8, F=8, N=8, act=salus.ACT_SILU, w_in_off=0, w_out_off=256, x_off=0, y_off=256, h_off=512)
GATED_GRAD = dict(job=0, M=4, K=8, F=8, N=8, act=salus.ACT_SILU, w_in_off=0, w_out_off=256, x_off=0, h_off=256, gu_off=512, dy_off=1024, dw_in_off=1280, dw_out_off=1536, work_off=2048)
DENSE = dict(job=0, M=4, K=8, N=8, act=salus.ACT_GELU, y_dtype=salus.F32, w_off=0, x_off=0, y_off=256)
DENSE_GRAD = dict(job=0, M=4, K=8, N=8, act=salus.ACT_NONE, w_off=0, x_off=0, dy_off=256, dw_off=512, work_off=1024)
TENSOR = dict(g_off=0, count=10, dtype=salus.BF16, wm_off=0, wb_off=256)
CLIP = dict(job=0, tensors=[TENSOR], max_norm=1.0, lr=0.1, norm_off=256, work_off=512)
MAKES = [(Pool.make_gated_descs, GATED), (Pool.make_gated_grad_descs, GATED_GRAD), (Pool.make_dense_descs, DENSE), (Pool.make_dense_grad_descs, DENSE_GRAD), (Pool.make_clip_descs, CLIP)]


@pytest.mark.parametrize("make,item", MAKES)
def test_values_arrive(make, item):
    descs, keep = make([item, item])
    assert len(descs) == 2
    for name, value in item.items():
        if name == "tensors":
            assert descs[1].n_tensors == 1 and all(getattr(descs[1].tensors[0], n) == v for n, v in TENSOR.items())
        else:
            assert getattr(descs[1], name) == pytest.approx(value)


@pytest.mark.parametrize("make,item", MAKES)
def test_numbers_that_do_not_fit(make, item):
    for name, value in item.items():
        if isinstance(value, int):
            bits = 64 if name.endswith("_off") else 32
            for bad in (2 ** bits + value, -2 ** bits + value, -2 ** (bits - 1) - 1):
                with pytest.raises(ValueError, match=name):
                    make([dict(item, **{name: bad})])


def test_tensor_numbers_that_do_not_fit():
    for name, value in TENSOR.items():
        for bad in (2 ** 64 + value, -2 ** 63 - 1):
            with pytest.raises(ValueError, match=name):
                Pool.make_clip_descs([dict(CLIP, tensors=[dict(TENSOR, **{name: bad})])])
            with pytest.raises(ValueError, match=name):
                salus.clip_work_bytes([dict(TENSOR, **{name: bad})])


@pytest.mark.parametrize("make,item", MAKES)
def test_unknown_names(make, item):
    with pytest.raises(ValueError, match="learning_rate"):
        make([dict(item, learning_rate=0.1)])


def test_unknown_names_of_tensors():
    with pytest.raises(ValueError, match="master_off"):
        Pool.make_clip_descs([dict(CLIP, tensors=[dict(TENSOR, master_off=0)])])


def test_work_bytes_of_numbers_that_do_not_fit():
    for ask in (salus.gated_grad_work_bytes, salus.dense_grad_work_bytes):
        assert ask(4, 8) > 0
        for M, N in ((2 ** 32 + 4, 8), (4, 2 ** 32 + 8), (-4, 8)):
            with pytest.raises(ValueError):
                ask(M, N)


def test_more_descriptors_than_there_are():
    """Refused by the binding, before the library reads them (a pool without device memory is enough for that)."""
    pool = Pool(None, 1 << 20)
    for make, item, run in ((Pool.make_dense_descs, DENSE, pool.grouped_dense_forward), (Pool.make_clip_descs, CLIP, pool.grouped_clip)):
        descs, keep = make([item])
        for n in (2, -1, 2 ** 32):
            with pytest.raises(ValueError):
                run(descs, n)
        assert run(descs, 0) == salus.OK
    pool.close()
