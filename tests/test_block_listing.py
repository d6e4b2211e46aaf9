"""The listing checks of the matrix-core instructions written in assembly (test_kernel_listing.py), for the product kernels with an
epilogue of their own, and what those kernels' waits count on (no GPU)."""
import pytest
import test_kernel_listing as K

pytestmark = K.pytestmark
# two result types, four kinds of operands
KERNELS = {"mxfp4_act_large_kernelI": 8, "mxfp4_act_tile_kernelILi2ELi4E": 8, "mxfp4_act_tile_kernelILi2ELi2E": 8, "mxfp4_act_twin_kernelI": 8}


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    found = {n: body for n, body in K.kernels(tmp_path_factory.mktemp("listing")).items() if any(k in n for k in KERNELS)}
    for kernel, count in KERNELS.items():
        assert sum(kernel in n for n in found) == count, kernel
    return found


def test_no_vector_instruction_writes_an_operand_right_before_a_matrix_core_instruction(listing):
    K.test_no_vector_instruction_writes_an_operand_right_before_a_matrix_core_instruction(listing)


def test_results_of_matrix_core_instructions_are_not_touched_too_early(listing):
    bad = []
    for name, body in listing.items():
        if "_large_" not in name:       # the others' instructions are builtins: the compiler keeps their distances
            continue
        before = K.predecessors(body)
        for n, ins in enumerate(body):
            if ins.is_mfma or ins.mnemonic.startswith("s_"):
                continue
            touched = ins.of(ins.operands)
            if touched:
                bad += [f"{name}: {ins.mnemonic} {ins.operands} at {ins.address:#x} behind {body[p].mnemonic} {body[p].operands}"
                        for p in K.within(body, before, n, 19, lambda i: i.is_mfma and i.registers(i.operands[0]) & touched)]
    assert not bad, f"{len(bad)} places, first ones:\n" + "\n".join(bad[:8])


@pytest.mark.parametrize("kernel,stores", [("mxfp4_act_large_kernelI", 64), ("mxfp4_act_tile_kernelILi2ELi4E", 32), ("mxfp4_act_tile_kernelILi2ELi2E", 16),
                                           ("mxfp4_act_twin_kernelI", 16)])
def test_a_tile_leaves_in_at_least_as_many_stores_as_the_kernels_count(listing, kernel, stores):
    # results: one store per pass of eight rows and 32-column slice, through the L2; in fp32 16 bytes, in bf16 8, where the kept pre-activations are as many again
    for name, body in listing.items():
        if kernel not in name:
            continue
        wide = sum(i.mnemonic == "buffer_store_dwordx4" and "sc1" in i.modifiers for i in body)
        narrow = sum(i.mnemonic == "buffer_store_dwordx2" and "sc1" in i.modifiers for i in body)
        assert (wide, narrow) == ((0, 2 * stores) if "Lb1E" in name.split(kernel)[1][:8] else (stores, stores))
        assert not any(i.mnemonic.startswith("scratch_") for i in body)
