// The recorder of launches (hip_recorder.cpp), and of the orthogonalised update's launches the plan that each was given, as text: a line for the plan and one
// a group, names and values.
#define hipLaunchKernel recorded_launch
#include "hip_recorder.cpp"
#undef hipLaunchKernel
#include <sstream>
typedef int hipError_t;
typedef void* hipStream_t;
#include "muon.hpp"

static std::vector<std::string> g_plans;

extern "C" {

int hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t lds, void* stream) {
    const int e = recorded_launch(f, grid, block, args, lds, stream);
    if (e != 0) return e;
    const std::string name = g_names.count(f) ? g_names[f] : "?";
    std::ostringstream s;
    if (name.find("muon_") != std::string::npos || name.find("ns_") != std::string::npos) {
        const blstm::MuonPlan& p = *static_cast<const blstm::MuonPlan*>(args[0]);
        s << "n " << p.n << " tile " << p.tile << " exact " << p.exact << " sums_at " << p.sums_at << " diag_at " << p.diag_at << " part_at " << p.part_at << " bytes " << p.bytes << "\n";
        for (int i = 0; i < p.n; ++i) {
            const blstm::MuonGroup& g = p.g[i];
            s << "rows " << g.rows << " cols " << g.cols << " count " << g.count << " ortho " << g.ortho << " rp " << g.rp << " cp " << g.cp << " mp " << g.mp << " tall " << g.tall
              << " splits " << g.splits << " x0 " << g.x[0] << " x1 " << g.x[1] << " s " << g.s << " b " << g.b << " xplane " << g.xplane << " splane " << g.splane << " diag " << g.diag
              << " part " << g.part << " chunks " << g.chunks << " casts " << g.casts << " grams " << g.grams << " applies " << g.applies << "\n";
        }
    }
    g_plans.resize(g_launches.size());
    g_plans.back() = s.str();
    return 0;
}
const char* recorder_plan(int i) { return g_plans[i].c_str(); }

}
