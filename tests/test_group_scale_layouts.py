"""Shared-memory plans of the products with group scales, compiled out of the sources and checked without a GPU."""
import re

import csrc_util


def test_the_plan_of_the_tensor_memory_kernel_holds_every_form():
    """Plain weights (two converter groups) and group scales (three): all barriers inside the plan, whose place depends on nothing but the
    form, and no form fits an SM beside a rotation, whose tensor memory it could take."""
    wo, tc = csrc_util.source("sq_gemm_wo.cu"), csrc_util.source("sq_rotate_quant_tc.cu")
    head = wo[wo.index("wo_gemm_tmem_kernel(const __grid_constant__"):]
    own = head[:head.index("// ---")].replace("extern __shared__", "").replace("__shared__ uint64_t gs_bars[X::GS ? 2 * CG : 1];", "")
    assert "__shared__" not in own                    # plain weights have nothing beside the plan
    plain = set(re.findall(r"launch_wo_decode<([\d, ]+)>\(", wo))
    scaled = set(re.findall(r"launch_wo_decode<([\d, ]+), X>\(", wo))
    assert len(plain) == 5 and len(scaled) == 3
    first = lambda form: ", ".join(form.split(", ")[:3])
    code = (csrc_util.lines(tc, r"^constexpr int k(?:Max|Half)DynSmem.*$") + "\n" + csrc_util.block(tc, "struct RqLayout")
            + csrc_util.block(tc, "__host__ __device__ inline RqLayout rq_layout(") + "\n"
            + csrc_util.lines(tc, r"^constexpr int kAloneSmem.*$|^inline int rq_smem.*$") + "\n"
            + csrc_util.lines(wo, r"^constexpr int (?:WO_|WOD_|WP_).*$") + "\n"
            + csrc_util.block(wo, "template <int NT, int ST, int SS>\nstruct WoDecSmem") + """
template <int NT, int ST, int SS> void show(int groups) {
  using L = WoDecSmem<NT, ST, SS>;
  printf("form %d %d %d\\n", (L::OFF_TMEM - L::OFF_BAR) / 8 - (2 * ST + 2 * SS + 4), 2 * groups, L::DYN_BYTES);
}
int main() {
""" + "".join(f"  show<{first(f)}>(2);\n" for f in plain) + "".join(f"  show<{first(f)}>(3);\n" for f in scaled) + """
  for (int n2 = 64; n2 <= 128; n2 *= 2)
    for (int n1 = 1; n1 <= 128; ++n1)
      for (int form = 1; form <= 2; ++form) {
        printf("rotate %d\\n", rq_smem(rq_layout(n1, n2, kMaxDynSmem, true), form));
        printf("rotate %d\\n", rq_smem(rq_layout(n1, n2, kHalfDynSmem), form));
      }
}""")
    rows = csrc_util.run(code)
    smallest = min(int(r[1]) for r in rows if r[0] == "rotate")
    forms = [tuple(map(int, r[1:])) for r in rows if r[0] == "form"]
    assert len(forms) == 8
    for room, operand_barriers, size in forms:
        assert room >= operand_barriers
        assert size <= 227 * 1024 and size + smallest + 2 * 1024 > 228 * 1024
