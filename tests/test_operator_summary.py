"""The table of the sequence operators' kernels, from traces made up here."""
import csv

from paper_1907_06154_amd import profiling

ROWS = "_ZN4ssam12_GLOBAL__N_19scan_rowsIDF16bNS_9ScanShapeILi4ELi4EEELb{}EEEvNS0_10ScanParamsE"
BACK = "void ssam::(anonymous namespace)::scan_back<float, ssam::ScanShape<4, 8>, {}, {}>(ssam::(anonymous namespace)::BackParams)"
FILL = "void at::native::vectorized_elementwise_kernel<4, at::native::FillFunctor<float>, std::array<char*, 1ul> >(int, at::native::FillFunctor<float>)"
RANDOM = "void at::native::(anonymous namespace)::distribution_elementwise_grid_stride_kernel<float, 4>(long)"


def trace(folder, kernels):
    folder.mkdir()
    with open(folder / "c_kernel_trace.csv", "w", newline="") as f:
        w = csv.DictWriter(f, ["Kernel_Name", "Start_Timestamp", "End_Timestamp"])
        w.writeheader()
        for i, (name, us) in enumerate(kernels):
            w.writerow({"Kernel_Name": name, "Start_Timestamp": i * 10 ** 6, "End_Timestamp": i * 10 ** 6 + int(us * 1e3)})


def test_every_kernel_of_a_call_is_listed(tmp_path):
    call = [(FILL, 4.5), (FILL, 4.5), (ROWS.format(0), 12), (ROWS.format(1), 15), (BACK.format("false", "true"), 13), (BACK.format("true", "false"), 43)]
    trace(tmp_path / "case", [(RANDOM, 99), (FILL, 7)] * 3 + call * profiling.OPERATE_CALLS)
    profiling.operator_summary(str(tmp_path), str(tmp_path / "out.md"))
    lines = [[c.strip() for c in line.split("|")[2:5]] for line in open(tmp_path / "out.md") if line.startswith("| case |") and "kernel" not in line]
    assert sorted(lines) == sorted([["`scan_rows` bf16 4 x 4, what the pieces add", "1", "12.0"], ["`scan_rows` bf16 4 x 4, everything", "1", "15.0"],
                                    ["`scan_back` fp32 4 x 8, what the pieces add", "1", "13.0"], ["`scan_back` fp32 4 x 8, everything", "1", "43.0"],
                                    ["torch: fill", "2", "4.5"]])
